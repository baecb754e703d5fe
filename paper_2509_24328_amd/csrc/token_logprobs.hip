// sv_token_logprobs: log-probabilities of given tokens, with normaliser, entropy, rank and the
// most probable alternatives.  sv_token_logprobs_grad: log-probability and entropy with the
// gradient of a weighted sum of them.
//
// One workgroup per logit row.  With y = z L - C (L = fl32(log2(e) / T), C a whole number near the row's
// largest z L) the row is reduced to S = sum 2^y and W = sum 2^y y, from which
//   lse = (C + log2 S) ln 2,  H = (log2 S - W / S) ln 2,  p_v = 2^y_v / S,
// so nothing is subtracted that is large against the result.  C is one number per wavefront while
// it sweeps: a whole one, so that raising it scales the sums exactly, and raised only when a logit
// lies more than kSlack above it, which after the first vectors is rare.
#include "sv_device.hpp"
#include "sv_host.hpp"

namespace sv {

constexpr float kSlack = 8.f;          // 2^y may be as large as 2^8: of no account for fp32 terms and fp64 sums
constexpr float kLowY = -200.f;        // 2^y is 0 in fp32 below: stands in for -inf where 2^y is multiplied by y

// Sums of one lane over its vectors; c is the wavefront's.
struct RowSums {
  float c, limit;     // reference; logits above the limit raise it
  float m;            // largest logit of the lane
  int best;           // the first of its vectors that holds it (where alternatives are asked for)
  double s, w;        // sum 2^y, sum 2^y y
  int ahead;          // entries before the token in the order of the alternatives

  __device__ __forceinline__ void init(float L) { c = kRefFloor; limit = c / L; m = -INFINITY; s = w = 0; best = 0; ahead = 0; }

  // (all lanes of the wavefront)
  __device__ __forceinline__ void raise(float largest, float L) {
    const float cn = whole_reference(wave_max_f32(largest), L);
    const float by = exp2_fast(c - cn);                 // a power of two, or 0
    w = (w + (double)(c - cn) * s) * (double)by;
    s *= (double)by;
    c = cn;
    limit = (cn + kSlack) / L;
  }
  static __device__ __forceinline__ float whole_reference(float m, float L) { return __builtin_ceilf(ref_of(m, L)); }
};

// What the workgroup knows of a row after the sweep.
struct RowTotals {
  float m, c;
  double s, w;
  int ahead;
  __device__ __forceinline__ bool bad() const { return !(s > 0.0) || !isfinite(s) || !isfinite(m) || c > kRefCeil; }
  __device__ __forceinline__ double log2_s() const { return log2(s); }
  __device__ __forceinline__ double lse(const Scale& sc) const {
    return ((double)c + log2_s()) * kLn2 - sc.tau1 * ((double)m * sc.inv_t);
  }
  __device__ __forceinline__ double entropy() const { return fmax(0.0, (log2_s() - w / s) * kLn2); }
};

template <int DT> __device__ __forceinline__ u32x4 no_mass() {
  const uint32_t v = DT == DT_F32 ? 0xff800000u : 0xff80ff80u;     // -inf
  return u32x4{v, v, v, v};
}

// Vector i of a row of V entries; the one past the last whole vector holds the entries left over.
template <int DT>
__device__ __forceinline__ u32x4 load_row_vec(const void* row, int V, int i) {
  constexpr int EPV = Elem<DT>::per_vec;
  const int nvec = V / EPV;
  if (i < nvec) return load_vec(row, i);
  u32x4 q = no_mass<DT>();
  for (int j = 0; j < V - i * EPV; ++j) {              // (negative past the row: no entry)
    if constexpr (DT == DT_F32) {
      q[j] = reinterpret_cast<const uint32_t*>(row)[i * EPV + j];
    } else {
      const uint32_t h = reinterpret_cast<const uint16_t*>(row)[i * EPV + j];
      q[j >> 1] = (j & 1) ? ((q[j >> 1] & 0x0000ffffu) | (h << 16)) : ((q[j >> 1] & 0xffff0000u) | h);
    }
  }
  return q;
}

// Adds U vectors of a lane (i, i + step, ...).  All lanes of the wavefront.
template <int DT, int U, bool ENT, bool TOP>
__device__ __forceinline__ void add_vectors(const u32x4 (&q)[U], int i, int step, float L, float zt, int token,
                                            RowSums& r) {
  constexpr int EPV = Elem<DT>::per_vec;
  float f[U][EPV];
  float gm = -INFINITY;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    unpack<DT>(q[u], f[u]);
    float vm = f[u][0];
#pragma unroll
    for (int j = 1; j + 1 < EPV; j += 2) vm = fmaxf(fmaxf(vm, f[u][j]), f[u][j + 1]);
    vm = fmaxf(vm, f[u][EPV - 1]);
    gm = fmaxf(gm, vm);
    if (TOP && vm > r.m) {
      r.m = vm;
      r.best = i + u * step;
    }
  }
  if (__any(gm > r.limit)) r.raise(gm, L);
  if (!TOP) r.m = fmaxf(r.m, gm);
  if (__any(gm >= zt)) {                               // (NaN without a token: never)
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < EPV; ++j)
        r.ahead += f[u][j] > zt || (f[u][j] == zt && (i + u * step) * EPV + j < token) ? 1 : 0;
  }
  float s = 0.f, w = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float e[EPV], ey[EPV];
#pragma unroll
    for (int j = 0; j < EPV; ++j) {
      const float y = __builtin_fmaf(f[u][j], L, -r.c);
      e[j] = exp2_fast(y);
      if (ENT) ey[j] = e[j] * fmaxf(y, kLowY);
    }
#pragma unroll
    for (int h = 1; h < EPV; h <<= 1)
#pragma unroll
      for (int j = 0; j < EPV; j += 2 * h) {
        e[j] += e[j + h];
        if (ENT) ey[j] += ey[j + h];
      }
    s += e[0];
    if (ENT) w += ey[0];
  }
  r.s += (double)s;
  if (ENT) r.w += (double)w;
}

struct RowScratch {
  double s[16], w[16];
  float m[16], c[16];
  int ahead[16];
};

// Sums of the workgroup, in every thread.
__device__ __forceinline__ RowTotals fold_row(const RowSums& r, RowScratch& sm) {
  const int wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
  const double s = wave_sum_f64(r.s), w = wave_sum_f64(r.w);
  const float m = wave_max_f32(r.m);
  const int ahead = __builtin_amdgcn_readlane(wave_scan_i32(r.ahead), kWave - 1);
  if ((threadIdx.x & 63) == 0) {
    sm.s[wave] = s; sm.w[wave] = w; sm.m[wave] = m; sm.c[wave] = r.c; sm.ahead[wave] = ahead;
  }
  __syncthreads();
  RowTotals t = {-INFINITY, kRefFloor, 0.0, 0.0, 0};
  for (int i = 0; i < nw; ++i) { t.m = fmaxf(t.m, sm.m[i]); t.c = fmaxf(t.c, sm.c[i]); }
  for (int i = 0; i < nw; ++i) {
    const float down = sm.c[i] - t.c;
    const double by = (double)exp2_fast(down);
    t.s += sm.s[i] * by;
    t.w += (sm.w[i] + (double)down * sm.s[i]) * by;
    t.ahead += sm.ahead[i];
  }
  return t;
}

// Sweep of a row by a workgroup of NT lanes; r keeps the lane's own part.
template <int DT, int NT, bool ENT, bool TOP>
__device__ __forceinline__ RowTotals sweep_row(const void* row, int V, float L, float zt, int token, RowSums& r,
                                               RowScratch& sm) {
  constexpr int EPV = Elem<DT>::per_vec, U = 4;
  const int n = (V + EPV - 1) / EPV;
  r.init(L);
  for (int i0 = 0; i0 < n; i0 += U * NT) {             // (the same number of rounds in every lane)
    u32x4 q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * NT + (int)threadIdx.x;
      q[u] = i < n ? load_row_vec<DT>(row, V, i) : no_mass<DT>();
    }
    add_vectors<DT, U, ENT, TOP>(q, i0 + (int)threadIdx.x, NT, L, zt, token, r);
  }
  return fold_row(r, sm);
}

struct ScoreArgs {
  const void* z;
  long long stride;                  // elements from row to row
  const int32_t* offsets;            // nullable: packed rows
  int n_rows;
  const int32_t* tokens;             // nullable
  int P, V, n_top;
  Scale sc;
  float *logprob, *lse, *entropy;    // nullable, like the rest
  int32_t *rank, *top_token;
  float* top_logprob;
  uint32_t* flags;
};

// Value in the order of the logits as a whole number (no NaN); -0 like 0.
__device__ __forceinline__ uint32_t ordered(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const uint64_t o = __shfl_xor(v, d, kWave);
    v = o > v ? o : v;
  }
  return v;
}

// A position without a row: nothing asked for, or nothing to be had.
__device__ __forceinline__ void write_blank(const ScoreArgs& a, long long at, bool bad) {
  const float x = bad ? __builtin_nanf("") : 0.f;
  for (int r = threadIdx.x; r < a.n_top; r += blockDim.x) {
    a.top_token[at * a.n_top + r] = -1;
    a.top_logprob[at * a.n_top + r] = bad ? x : -INFINITY;
  }
  if (threadIdx.x != 0) return;
  if (a.logprob) a.logprob[at] = x;
  if (a.lse) a.lse[at] = x;
  if (a.entropy) a.entropy[at] = x;
  if (a.rank) a.rank[at] = 0;
  if (a.flags) a.flags[at] = bad ? SV_FLAG_BAD_ROW : 0;
}

// The n first entries of a row in the order by value and, among equal ones, by token.  After the sweep every lane knows
// its largest entry.  The n lanes that are first by (value, vector) hold the n first entries: an entry of any
// other lane has n before it.  So the lanes are ranked (only those that a bound lets through, which each
// wavefront forms from its own), the n lanes' vectors read again, and what is not behind the n-th lane's best ranked
// in turn.  Ranks by counting: the keys are distinct, and about n lanes and little more than n entries are
// left.  The sweep pays two instructions a vector for this, whatever the row holds.
constexpr int kCandidates = 1024;

template <int NT>
struct TopScratch {
  uint64_t lanes[NT], first[SV_TOP_MAX], found[kCandidates];
  float bound[NT / kWave];
  int n_lanes, n_found;
};

template <int DT, int NT, class Emit>
__device__ __forceinline__ void alternatives(const void* row, int V, float L, int n, float best, int best_vec,
                                             TopScratch<NT>& sm, Emit&& emit) {
  constexpr int EPV = Elem<DT>::per_vec, kWaves = NT / kWave;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n_vec = (V + EPV - 1) / EPV;
  if (!(best * L >= kRefFloor)) best = -INFINITY;      // nothing with mass
  // n lanes at least are not below the lowest, over the wavefronts, of their n / kWaves-th lanes
  float left = best, low = 0.f;
  for (int j = 0; j < n; j += kWaves) {
    low = wave_max_f32(left);
    if (lane == __builtin_ctzll(__ballot(left == low))) left = -INFINITY;
  }
  if (lane == 0) sm.bound[wave] = low;
  if (tid == 0) sm.n_lanes = sm.n_found = 0;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) low = fminf(low, sm.bound[w]);
  if (best >= low && best > -INFINITY)
    sm.lanes[atomicAdd(&sm.n_lanes, 1)] = (uint64_t)ordered(best) << 32 | (uint32_t)~best_vec;
  __syncthreads();
  const int n_lanes = sm.n_lanes, n_first = min(n, n_lanes);
  if (tid < n_lanes) {
    const uint64_t key = sm.lanes[tid];
    int rank = 0;
    for (int m = 0; m < n_lanes; ++m) rank += sm.lanes[m] > key;
    if (rank < n) sm.first[rank] = key;
  }
  __syncthreads();
  const uint64_t last = n_lanes >= n ? sm.first[n - 1] : 0;
  const float last_z = last ? from_ordered((uint32_t)(last >> 32)) : -INFINITY;
  const int last_vec = last ? (int)~(uint32_t)last : V;
  const int per_lane = (n_vec + NT - 1) / NT;
  auto visit = [&](auto&& take) {                      // the entries of the first lanes that may be among the n
    for (int p = tid; p < n_first * per_lane; p += NT) {
      const int i = (int)~(uint32_t)sm.first[p % n_first] % NT + p / n_first * NT;
      if (i >= n_vec) continue;
      float f[EPV];
      unpack<DT>(load_row_vec<DT>(row, V, i), f);
#pragma unroll
      for (int j = 0; j < EPV; ++j)
        if ((f[j] > last_z || (f[j] == last_z && i <= last_vec)) && f[j] * L >= kRefFloor)
          take((uint64_t)ordered(f[j]) << 32 | (uint32_t)~(i * EPV + j));
    }
  };
  visit([&](uint64_t key) {
    const int at = atomicAdd(&sm.n_found, 1);
    if (at < kCandidates) sm.found[at] = key;
  });
  __syncthreads();
  const int n_found = sm.n_found;
  if (n_found <= kCandidates) {
    for (int t = tid; t < n_found; t += NT) {
      const uint64_t key = sm.found[t];
      int rank = 0;
      for (int m = 0; m < n_found; ++m) rank += sm.found[m] > key;
      if (rank < n) emit(rank, key);
    }
    if (tid < n && tid >= n_found) emit(tid, 0);
    return;
  }
  // large entries that all lie in few lanes: the largest one below the one before, n times
  uint64_t before = ~0ull;
  for (int r = 0; r < n; ++r) {
    uint64_t key = 0;
    visit([&](uint64_t k) { key = k < before && k > key ? k : key; });
    key = wave_max_u64(key);
    if (lane == 0) sm.lanes[wave] = key;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) key = sm.lanes[w] > key ? sm.lanes[w] : key;
    __syncthreads();
    if (tid == 0) emit(r, key);
    before = key;
  }
}

template <int DT, int NT, bool ENT, bool TOP>
__global__ __launch_bounds__(NT) void token_logprobs_kernel(const ScoreArgs a) {
  __shared__ RowScratch sm;
  const long long at = blockIdx.x;
  const int V = a.V;
  int token = -1;
  if (a.tokens) {
    token = a.tokens[at];
    if (token == -1) return write_blank(a, at, false);
  }
  long long at_row = at;
  if (a.offsets) {
    const int b = (int)(at / a.P), i = (int)(at % a.P);
    const long long lo = a.offsets[b], hi = a.offsets[b + 1];
    if (i >= hi - lo) return write_blank(a, at, false);
    at_row = lo + i;
    if (at_row < 0 || at_row >= a.n_rows) return write_blank(a, at, true);
  }
  const void* row = static_cast<const char*>(a.z) + (size_t)at_row * (size_t)a.stride * Elem<DT>::bytes;
  const bool given = token >= 0 && token < V;
  const float zt = given ? load_elem<DT>(row, token) : __builtin_nanf("");
  RowSums r;
  const RowTotals t = sweep_row<DT, NT, ENT, TOP>(row, V, a.sc.L, zt, token, r, sm);
  if (t.bad()) return write_blank(a, at, true);
  const double lse = t.lse(a.sc);
  auto logprob_of = [&](float z) {
    return z * a.sc.L < kRefFloor ? -INFINITY : (float)((double)z * a.sc.inv_t - lse);
  };
  if (threadIdx.x == 0) {
    if (a.logprob) a.logprob[at] = given ? logprob_of(zt) : __builtin_nanf("");
    if (a.lse) a.lse[at] = (float)lse;
    if (a.entropy) a.entropy[at] = (float)t.entropy();
    if (a.rank) a.rank[at] = given ? 1 + t.ahead : 0;
    if (a.flags) a.flags[at] = a.tokens && !given ? SV_FLAG_BAD_TOKEN : 0;
  }
  if constexpr (TOP) {
    __shared__ TopScratch<NT> top;
    alternatives<DT, NT>(row, V, a.sc.L, a.n_top, r.m, r.best, top, [&](int rank, uint64_t key) {
      a.top_token[at * a.n_top + rank] = key ? (int)~(uint32_t)key : -1;
      a.top_logprob[at * a.n_top + rank] = key ? logprob_of(from_ordered((uint32_t)(key >> 32))) : -INFINITY;
    });
  }
}

constexpr int kGradThreads = 1024;

template <int DT, bool ENT>
void launch_score(const ScoreArgs& a, long long rows, hipStream_t st) {
  const dim3 grid((unsigned)rows);
  if (a.n_top > 0) hipLaunchKernelGGL((token_logprobs_kernel<DT, 1024, ENT, true>), grid, dim3(1024), 0, st, a);
  else hipLaunchKernelGGL((token_logprobs_kernel<DT, 1024, ENT, false>), grid, dim3(1024), 0, st, a);
}

struct GradArgs {
  const void* z;
  void* dz;
  long long stride, dz_stride;
  const int32_t* tokens;
  const float *g_logprob, *g_entropy;
  float *logprob, *entropy;
  uint32_t* flags;
  int V;
  Scale sc;
};

// Vector i of a row of V entries, the counterpart of load_row_vec.
template <int DT>
__device__ __forceinline__ void store_row_vec(void* row, int V, int i, const float (&f)[Elem<DT>::per_vec]) {
  constexpr int EPV = Elem<DT>::per_vec;
  u32x4 q;
  if constexpr (DT == DT_F32) {
    q = u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  } else {
    q = u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
  }
  if (i < V / EPV) {
    reinterpret_cast<u32x4_row*>(row)[i] = q;
    return;
  }
  for (int j = 0; j < V - i * EPV; ++j) {
    if constexpr (DT == DT_F32) reinterpret_cast<uint32_t*>(row)[i * EPV + j] = q[j];
    else reinterpret_cast<uint16_t*>(row)[i * EPV + j] = (uint16_t)(q[j >> 1] >> (16 * (j & 1)));
  }
}

template <int DT, bool ENT>
__global__ __launch_bounds__(kGradThreads) void token_logprobs_grad_kernel(const GradArgs a) {
  constexpr int EPV = Elem<DT>::per_vec;
  __shared__ RowScratch sm;
  const long long at = blockIdx.x;
  const int V = a.V, token = a.tokens[at];
  const void* row = static_cast<const char*>(a.z) + (size_t)at * (size_t)a.stride * Elem<DT>::bytes;
  char* out = static_cast<char*>(a.dz) + (size_t)at * (size_t)a.dz_stride * Elem<DT>::bytes;
  auto fill = [&](float x) {
    float f[EPV];
#pragma unroll
    for (int j = 0; j < EPV; ++j) f[j] = x;
    for (int i = threadIdx.x; i * EPV < V; i += blockDim.x) store_row_vec<DT>(out, V, i, f);
  };
  if (token == -1) {
    fill(0.f);
    if (threadIdx.x != 0) return;
    if (a.logprob) a.logprob[at] = 0.f;
    if (a.entropy) a.entropy[at] = 0.f;
    if (a.flags) a.flags[at] = 0;
    return;
  }
  const bool given = token >= 0 && token < V;
  const float zt = given ? load_elem<DT>(row, token) : __builtin_nanf("");
  RowSums r;
  const RowTotals t = sweep_row<DT, kGradThreads, ENT, false>(row, V, a.sc.L, __builtin_nanf(""), -1, r, sm);
  const bool bad = t.bad();
  if (threadIdx.x == 0) {
    const double x = bad || !given ? (double)__builtin_nanf("")
                                   : (zt * a.sc.L < kRefFloor ? -INFINITY : (double)zt * a.sc.inv_t - t.lse(a.sc));
    if (a.logprob) a.logprob[at] = (float)x;
    if (a.entropy) a.entropy[at] = bad ? __builtin_nanf("") : (float)t.entropy();
    if (a.flags) a.flags[at] = (bad ? SV_FLAG_BAD_ROW : 0) | (given ? 0 : SV_FLAG_BAD_TOKEN);
  }
  if (bad || !given) return fill(__builtin_nanf(""));
  // dz_v = 2^y (a0 + a1 y), and g / T more at the token:  log p = (y - log2 S) ln 2
  const double g = (double)a.g_logprob[at], h = ENT && a.g_entropy ? (double)a.g_entropy[at] : 0.0;
  const double inv_s = a.sc.inv_t / t.s;
  const float a1 = (float)(-inv_s * h * kLn2);
  const float a0 = (float)(-inv_s * (g + h * (ENT ? t.entropy() - t.log2_s() * kLn2 : 0.0)));
  const float at_token = (float)(g * a.sc.inv_t);
  for (int i = threadIdx.x; i * EPV < V; i += blockDim.x) {
    float f[EPV];
    unpack<DT>(load_row_vec<DT>(row, V, i), f);
#pragma unroll
    for (int j = 0; j < EPV; ++j) {
      const float y = __builtin_fmaf(f[j], a.sc.L, -t.c);
      f[j] = exp2_fast(y) * (ENT ? __builtin_fmaf(fmaxf(y, kLowY), a1, a0) : a0);
    }
    if (token / EPV == i) {
#pragma unroll
      for (int j = 0; j < EPV; ++j) f[j] += token % EPV == j ? at_token : 0.f;
    }
    store_row_vec<DT>(out, V, i, f);
  }
}

}  // namespace sv

extern "C" int sv_token_logprobs(const void* z, int64_t z_stride, const int32_t* t_offsets_or_null, int n_rows,
                                 const int32_t* tokens_or_null, int B, int P, int V, int dtype, float temperature,
                                 int n_top, float* logprob_or_null, float* lse_or_null, float* entropy_or_null,
                                 int32_t* rank_or_null, int32_t* top_token_or_null, float* top_logprob_or_null,
                                 uint32_t* flags_or_null, sv_stream_t stream) {
  using namespace sv;
  SV_REQUIRE(dtype == SV_F32 || dtype == SV_BF16, SV_ERR_DTYPE);
  SV_REQUIRE(B >= 0 && P >= 1 && V >= 1 && z_stride >= V && n_top >= 0, SV_ERR_INVALID_ARG);
  SV_REQUIRE(!t_offsets_or_null || n_rows >= 0, SV_ERR_INVALID_ARG);
  ScoreArgs a = {};
  SV_REQUIRE(scale_of(temperature, &a.sc), SV_ERR_INVALID_ARG);
  SV_REQUIRE(V <= (1 << 24) && n_top <= SV_TOP_MAX && (long long)B * P <= 0x7fffffffLL, SV_ERR_TOO_LARGE);
  if (B == 0) return SV_OK;
  SV_REQUIRE(z && (tokens_or_null || (!logprob_or_null && !rank_or_null)), SV_ERR_NULL);
  SV_REQUIRE(n_top == 0 || (top_token_or_null && top_logprob_or_null), SV_ERR_NULL);
  SV_REQUIRE(is_aligned(z, elem_bytes(dtype)) && is_aligned(t_offsets_or_null, 4) && is_aligned(tokens_or_null, 4) &&
                 is_aligned(logprob_or_null, 4) && is_aligned(lse_or_null, 4) && is_aligned(entropy_or_null, 4) &&
                 is_aligned(rank_or_null, 4) && is_aligned(top_token_or_null, 4) &&
                 is_aligned(top_logprob_or_null, 4) && is_aligned(flags_or_null, 4),
             SV_ERR_ALIGN);
  a.z = z; a.stride = z_stride; a.offsets = t_offsets_or_null; a.n_rows = n_rows; a.tokens = tokens_or_null;
  a.P = P; a.V = V; a.n_top = n_top;
  a.logprob = logprob_or_null; a.lse = lse_or_null; a.entropy = entropy_or_null; a.rank = rank_or_null;
  a.top_token = top_token_or_null; a.top_logprob = top_logprob_or_null; a.flags = flags_or_null;
  const long long rows = (long long)B * P;
  hipStream_t st = as_stream(stream);
  if (dtype == SV_F32) {
    if (entropy_or_null) launch_score<DT_F32, true>(a, rows, st);
    else launch_score<DT_F32, false>(a, rows, st);
  } else {
    if (entropy_or_null) launch_score<DT_BF16, true>(a, rows, st);
    else launch_score<DT_BF16, false>(a, rows, st);
  }
  return launch_status();
}

extern "C" int sv_token_logprobs_grad(const void* z, int64_t z_stride, const int32_t* tokens, int rows, int V,
                                      int dtype, float temperature, const float* g_logprob,
                                      const float* g_entropy_or_null, float* logprob_or_null, float* entropy_or_null,
                                      void* dz, int64_t dz_stride, uint32_t* flags_or_null, sv_stream_t stream) {
  using namespace sv;
  SV_REQUIRE(dtype == SV_F32 || dtype == SV_BF16, SV_ERR_DTYPE);
  SV_REQUIRE(rows >= 0 && V >= 1 && z_stride >= V && dz_stride >= V, SV_ERR_INVALID_ARG);
  SV_REQUIRE(dz != z || dz_stride == z_stride, SV_ERR_INVALID_ARG);
  GradArgs a = {};
  SV_REQUIRE(scale_of(temperature, &a.sc), SV_ERR_INVALID_ARG);
  SV_REQUIRE(V <= (1 << 24), SV_ERR_TOO_LARGE);
  if (rows == 0) return SV_OK;
  SV_REQUIRE(z && dz && tokens && g_logprob, SV_ERR_NULL);
  SV_REQUIRE(is_aligned(z, elem_bytes(dtype)) && is_aligned(dz, elem_bytes(dtype)) && is_aligned(tokens, 4) &&
                 is_aligned(g_logprob, 4) && is_aligned(g_entropy_or_null, 4) && is_aligned(logprob_or_null, 4) &&
                 is_aligned(entropy_or_null, 4) && is_aligned(flags_or_null, 4),
             SV_ERR_ALIGN);
  a.z = z; a.dz = dz; a.stride = z_stride; a.dz_stride = dz_stride; a.tokens = tokens;
  a.g_logprob = g_logprob; a.g_entropy = g_entropy_or_null; a.logprob = logprob_or_null; a.entropy = entropy_or_null;
  a.flags = flags_or_null; a.V = V;
  const bool ent = entropy_or_null || g_entropy_or_null;
  const dim3 grid((unsigned)rows), block(kGradThreads);
  hipStream_t st = as_stream(stream);
  if (dtype == SV_F32) {
    if (ent) hipLaunchKernelGGL((token_logprobs_grad_kernel<DT_F32, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((token_logprobs_grad_kernel<DT_F32, false>), grid, block, 0, st, a);
  } else {
    if (ent) hipLaunchKernelGGL((token_logprobs_grad_kernel<DT_BF16, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((token_logprobs_grad_kernel<DT_BF16, false>), grid, block, 0, st, a);
  }
  return launch_status();
}
