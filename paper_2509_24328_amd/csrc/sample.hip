// sv_sample: a token of every row under temperature, top-k, top-p and min-p, from a given random number.
//
// One workgroup per row.  The warps only concern the upper tail of a row, so they are settled on a short list of its largest entries:
//   sweep 1  the row's maximum m and the maxima of the 1024 lanes, which are distinct entries of the row (without a K: the
//            row's mass as well)
//   list     the entries not below some value tau, sorted.  tau is the K-th largest lane maximum (at least K entries of the row are as
//            large), or a guess for a nucleus, or what min-p says
//   settle   the K-th value; masses down the list until they reach P
// A list that is too long or does not reach as far as the warps do is narrowed from both sides: a sweep counts (and weighs) what lies
// above a value in between, until the stretch that holds the cutoff fits the list or is one value.
// The token is then found among the kept entries of the list, or, where there are too many of them, from the masses of pieces of
// the row and the entries of one piece.
// Weights are fp64 (2^x as a polynomial: an error of 1e-15, where float32 exponentials would make 1 row in 300 of a flat 152064-entry
// distribution draw another token), and every sum has an order that the sizes fix.
#include "sv_device.hpp"
#include "sv_host.hpp"

namespace sv {

constexpr int kDrawThreads = 1024;
constexpr int kDrawWaves = kDrawThreads / kWave;
constexpr int kList = 2048;              // entries of the list
constexpr int kPieceVecs = 8;            // vectors of a lane in a piece: 4096 bfloat16 or 2048 float32 entries
constexpr int kNucleusRank = 256;        // first guess of a nucleus: the entries above this many lane maxima

struct SampleArgs {
  const char* z;
  int64_t z_stride;                      // bytes
  int V, top_k;                          // 0: no K
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
    const int t = threadIdx.x;
    const double w0 = 2 * t < n ? weight(list_value(2 * t)) : 0.0, w1 = 2 * t + 1 < n ? weight(list_value(2 * t + 1)) : 0.0;
    double total;
    const double incl = block_scan(w0 + w1, &total, sh);
    if (2 * t < n) sh.cum[2 * t] = before + (incl - w1);
    if (2 * t + 1 < n) sh.cum[2 * t + 1] = before + incl;
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

  // The entries of sh.key[0 .. n) by ascending token, and the one that holds u W; W.
  __device__ __forceinline__ float draw_listed(int n, double u, int* token, double* total) {
    // keys by token: the lower halves descend with it
    for (int i = threadIdx.x; i < n; i += kDrawThreads) sh.key[i] = (sh.key[i] << 32) | (sh.key[i] >> 32);
    __syncthreads();
    sort(n);
    const int t = threadIdx.x;
    auto value = [&](int i) { return key_float((uint32_t)sh.key[i]); };
    const double w0 = 2 * t < n ? weight(value(2 * t)) : 0.0, w1 = 2 * t + 1 < n ? weight(value(2 * t + 1)) : 0.0;
    double W;
    const double incl = block_scan(w0 + w1, &W, sh);
    if (t == 0) sh.hit = 0x7fffffff;
    if (t == 0) sh.n = -1;
    __syncthreads();
    const double at = u * W;
    if (w0 > 0.0 && incl - w1 > at) atomicMin(&sh.hit, 2 * t);
    else if (w1 > 0.0 && incl > at) atomicMin(&sh.hit, 2 * t + 1);
    if (w1 > 0.0) atomicMax(&sh.n, 2 * t + 1);
    else if (w0 > 0.0) atomicMax(&sh.n, 2 * t);
    __syncthreads();
    const int i = sh.hit < n ? sh.hit : sh.n;            // (u W rounded up to W: the last one)
    *token = (int)~(uint32_t)(sh.key[i] >> 32);
    *total = W;
    return value(i);
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
    const int t = threadIdx.x;
    const double w0 = 2 * t < groups ? mass[2 * t] : 0.0, w1 = 2 * t + 1 < groups ? mass[2 * t + 1] : 0.0;
    double W;
    const double incl = block_scan(w0 + w1, &W, sh);
    const double at = u * W;
    if (t == 0) { sh.hit = 0x7fffffff; sh.n = 0; }
    __syncthreads();
    if (w0 > 0.0 && incl - w1 > at) atomicMin(&sh.hit, 2 * t);
    else if (w1 > 0.0 && incl > at) atomicMin(&sh.hit, 2 * t + 1);
    if (w1 > 0.0) atomicMax(&sh.n, 2 * t + 1);
    else if (w0 > 0.0) atomicMax(&sh.n, 2 * t);
    __syncthreads();
    const int gI = sh.hit < groups ? sh.hit : sh.n;
    if (2 * t == gI) sh.out_d[0] = incl - w1 - w0;       // the mass before the group
    if (2 * t + 1 == gI) sh.out_d[0] = incl - w1;
    __syncthreads();
    if (wave == 0) {                                     // one wavefront, vector by vector of 64 lanes
      double before = sh.out_d[0];
      int found = -1, last = -1;
      const int nvec = a.V / EPV;
      for (int p = gI * group; p < min((gI + 1) * group, pieces) && found < 0; ++p)
        for (int j = 0; j < kPieceVecs && found < 0; ++j) {
          const int64_t i = ((int64_t)p * kPieceVecs + j) * kWave + lane;
          double w[EPV], s = 0.0;
#pragma unroll
          for (int e = 0; e < EPV; ++e) {
            const int64_t v = i * EPV + e;
            w[e] = i <= nvec && v < a.V ? kept_weight(load_elem<DT>(row, (int)v), least) : 0.0;
            s += w[e];
          }
          const double incl_l = wave_scan_f64(s);
          double run = before + (incl_l - s);
          int mine = -1, mine_last = -1;
#pragma unroll
          for (int e = 0; e < EPV; ++e) {
            run += w[e];
            if (w[e] > 0.0) {
              mine_last = (int)(i * EPV + e);
              if (mine < 0 && run > at) mine = mine_last;
            }
          }
          const uint64_t hits = __ballot(mine >= 0), any = __ballot(mine_last >= 0);
          if (hits) found = __builtin_amdgcn_readlane(mine, __builtin_ctzll(hits));
          if (any) last = __builtin_amdgcn_readlane(mine_last, 63 - __builtin_clzll(any));
          before += lane_f64(incl_l, kWave - 1);
        }
      if (lane == 0) sh.out_i[0] = found >= 0 ? found : last;
    }
    __syncthreads();
    *token = sh.out_i[0];
    *total = W;
    return load_elem<DT>(row, *token);
  }
};

template <int DT>
__global__ void __launch_bounds__(kDrawThreads) sample_kernel(SampleArgs a) {
  constexpr int EPV = Elem<DT>::per_vec;
  __shared__ DrawShared sh;
  const int64_t r = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  Draw<DT> d{a, a.z + r * a.z_stride, sh, 0.0};
  // sweep 1
  float mine = -INFINITY;
  bool nan = false;
  d.each([&](const float (&x)[EPV], int, int n) {
#pragma unroll
    for (int e = 0; e < EPV; ++e) {
      mine = fmaxf(mine, x[e]);
      nan |= x[e] != x[e];
    }
  });
  const float wave_top = wave_max_f32(nan ? INFINITY : mine);
  if (lane == 0) sh.wave_u[wave] = __float_as_uint(wave_top);
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < kDrawWaves; ++w) top = fmaxf(top, __uint_as_float(sh.wave_u[w]));
  __syncthreads();
  double u = a.u[r];
  const double y = (double)top * a.scale;
  if (!(y >= (double)kRefFloor && y <= (double)kRefCeil) || u != u) {
    if (tid == 0) {
      a.token[r] = -1;
      if (a.logprob) a.logprob[r] = NAN;
      if (a.flags) a.flags[r] = SV_FLAG_BAD_ROW;
    }
    return;
  }
  u = fmin(fmax(u, 0.0), 1.0 - 0x1p-53);
  d.m = (double)top;

  const bool use_k = a.top_k > 0 && a.top_k < a.V, use_p = a.top_p < 1.0, use_min = a.min_log2 > -INFINITY;
  int token = 0;
  double W = 0.0;
  float z = 0.f;
  bool done = false;
  uint32_t least = order_key(-INFINITY);                // keys below it are dropped
  if (use_k || use_p || use_min) {
    double all = 0.0;
    int count;
    if (use_p && !use_k) d.above(least, true, count, all);
    // tau
    uint32_t tau = least, min_key = least;
    if (use_min) {
      // (a step of a float32 below, where the weight is looked at again)
      const double zm = d.m + a.min_log2 / a.scale;
      min_key = order_key((float)zm) - 2;
      if (min_key < least || zm < -3e38) min_key = least;
    }
    const int want = use_k ? a.top_k : (use_p ? kNucleusRank : 0);
    if (want > 0 && want <= kDrawThreads) {
      const uint32_t key = order_key(mine);
      uint32_t t = 0;
      for (int bit = 31; bit >= 16; --bit) {             // the want-th largest lane maximum, its upper sixteen bits
        const uint32_t probe = t | (1u << bit);
        if (__syncthreads_count(key >= probe) >= want) t = probe;
      }
      tau = max(t, least);
    }
    if (!use_k) tau = max(tau, min_key);                 // (the K-th value may lie below what min-p keeps)
    const int n = want > kDrawThreads ? kList + 1 : d.list(tau, 0);
    bool settled = n <= kList;
    if (settled) {
      int keep = n;                                      // of the list, by value
      if (use_k) {
        if (n < a.top_k) settled = false;
        else {
          const uint32_t kth = (uint32_t)(sh.key[a.top_k - 1] >> 32);
          keep = a.top_k;
          // ties with the K-th
          for (int step = 1024; step > 0; step >>= 1)
            if (keep + step <= n && (uint32_t)(sh.key[keep + step - 1] >> 32) >= kth) keep += step;
        }
      }
      if (settled && use_p) {
        d.masses(keep, 0.0);
        const double target = a.top_p * (use_k ? sh.cum[keep - 1] : all);
        const int i = d.reach(keep, target);
        if (i < keep) {
          const uint32_t c = (uint32_t)(sh.key[i] >> 32);
          int k2 = i + 1;
          for (int step = 1024; step > 0; step >>= 1)
            if (k2 + step <= keep && (uint32_t)(sh.key[k2 + step - 1] >> 32) >= c) k2 += step;
          keep = k2;
        } else if (!use_k && !(use_min && tau <= min_key)) {
          settled = false;                               // the list does not reach as far as the nucleus
        }
      }
      if (settled && use_min) {
        int k2 = 0;                                      // entries whose weight is at least min_p
        for (int step = 2048; step > 0; step >>= 1)
          if (k2 + step <= keep && d.weight_log2(d.list_value(k2 + step - 1)) >= a.min_log2) k2 += step;
        keep = max(k2, 1);
        if (!use_k && !use_p && tau > min_key) settled = false;
      }
      __syncthreads();
      if (settled) {
        z = d.draw_listed(keep, u, &token, &W);
        done = true;
      }
    }
    if (!done) {
      if (use_k) {
        least = d.narrow(true, a.top_k, 0.0, order_key(-INFINITY), a.V, 0, 0, 0.0);
        if (use_p) d.above(least, true, count, all);
      }
      if (use_p) {
        int n_lo = count;
        least = d.narrow(false, 0, a.top_p * all, least, n_lo, 0, 0, 0.0);
      }
    }
  }
  if (!done) z = d.draw_swept(key_float(least), u, &token, &W);
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
  SampleArgs a{static_cast<const char*>(z), z_stride * e, V, top_k > 0 && top_k < V ? top_k : 0, kLog2e / (double)temperature, sc.inv_t,
               top_p < 1.f ? (double)top_p : 1.0, min_p > 0.f ? __builtin_log2((double)min_p) : -INFINITY, u, token, logprob_or_null,
               flags_or_null};
  in_launches(rows, kDrawThreads, [&](long long first, dim3 grid) {
    SampleArgs b = a;
    b.z += first * b.z_stride;
    b.u += first;
    b.token += first;
    if (b.logprob) b.logprob += first;
    if (b.flags) b.flags += first;
    if (dtype == SV_F32) hipLaunchKernelGGL(sample_kernel<DT_F32>, grid, dim3(kDrawThreads), 0, as_stream(stream), b);
    else hipLaunchKernelGGL(sample_kernel<DT_BF16>, grid, dim3(kDrawThreads), 0, as_stream(stream), b);
  });
  return launch_status();
}
