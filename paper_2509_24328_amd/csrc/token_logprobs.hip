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

constexpr int kAhead = 4;              // vectors of a lane under way
constexpr float kSlack = 8.f;          // 2^y may be as large as 2^8: of no account for fp32 terms and fp64 sums
constexpr float kLowY = -200.f;        // 2^y is 0 in fp32 below: stands in for -inf where 2^y is multiplied by y

// Sums of one lane over its vectors; c is the wavefront's.
struct RowSums {
  float c, limit;     // reference; logits above the limit raise it
  float m;            // largest logit of the lane
  int best;           // the first of its vectors that holds it (where alternatives are asked for)
  float sf, wf;       // sum 2^y, sum 2^y y of the last few vectors
  double s, w;        // of the vectors before those
  int ahead;          // entries before the token in the order of the alternatives

  __device__ __forceinline__ void init(float L) {
    c = kRefFloor; limit = c / L; m = -INFINITY; best = 0; sf = wf = 0.f; s = w = 0; ahead = 0;
  }
  __device__ __forceinline__ void flush() {
    s += (double)sf;
    w += (double)wf;
    sf = wf = 0.f;
  }
  // (all lanes of the wavefront)
  __device__ __forceinline__ void raise(float largest, float L) {
    const float cn = __builtin_ceilf(ref_of(wave_max_f32(largest), L));
    const float by = exp2_fast(c - cn);                 // a power of two, or 0
    flush();
    w = (w + (double)(c - cn) * s) * (double)by;
    s *= (double)by;
    c = cn;
    limit = (cn + kSlack) / L;
  }
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

template <int DT> __device__ __forceinline__ int vectors_of(int V) { return (V + Elem<DT>::per_vec - 1) / Elem<DT>::per_vec; }

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

// Adds vector i of a lane's.  All lanes of the wavefront.
template <int DT, bool ENT, bool TOP>
__device__ __forceinline__ void add_vector(const u32x4& q, int i, float L, float zt, int token, RowSums& r) {
  constexpr int EPV = Elem<DT>::per_vec;
  float f[EPV];
  unpack<DT>(q, f);
  float vm = f[0];
#pragma unroll
  for (int j = 1; j + 1 < EPV; j += 2) vm = fmaxf(fmaxf(vm, f[j]), f[j + 1]);
  vm = fmaxf(vm, f[EPV - 1]);
  if (__any(vm > r.limit)) r.raise(vm, L);
  if (TOP) {
    r.best = vm > r.m ? i : r.best;
  }
  r.m = fmaxf(r.m, vm);
  if (__any(vm >= zt)) {                               // (NaN without a token: never)
#pragma unroll
    for (int j = 0; j < EPV; ++j) r.ahead += f[j] > zt || (f[j] == zt && i * EPV + j < token) ? 1 : 0;
  }
  float e[EPV], w0 = r.wf, w1 = 0.f;
#pragma unroll
  for (int j = 0; j < EPV; ++j) {
    const float y = __builtin_fmaf(f[j], L, -r.c);
    e[j] = exp2_fast(y);
    if (ENT) (j & 1 ? w1 : w0) = __builtin_fmaf(e[j], fmaxf(y, kLowY), j & 1 ? w1 : w0);
  }
#pragma unroll
  for (int h = 1; h < EPV; h <<= 1)
#pragma unroll
    for (int j = 0; j < EPV; j += 2 * h) e[j] += e[j + h];
  r.sf += e[0];
  if (ENT) r.wf = w0 + w1;
}

struct RowScratch {
  double s[16], w[16];
  float m[16], c[16];
  int ahead[16];
};

// A wavefront's sums, for fold_row after the next barrier.
__device__ __forceinline__ void leave_row(const RowSums& r, RowScratch& sm) {
  const int wave = threadIdx.x >> 6;
  const double s = wave_sum_f64(r.s), w = wave_sum_f64(r.w);
  const float m = wave_max_f32(r.m);
  const int ahead = __builtin_amdgcn_readlane(wave_scan_i32(r.ahead), kWave - 1);
  if ((threadIdx.x & 63) == 0) {
    sm.s[wave] = s; sm.w[wave] = w; sm.m[wave] = m; sm.c[wave] = r.c; sm.ahead[wave] = ahead;
  }
}

// Sums of NT lanes, in every lane of the wavefronts that ask: a row of 16 lanes folds, one wavefront's sums a lane.
template <int NT>
__device__ __forceinline__ RowTotals fold_row(const RowScratch& sm) {
  const int i = threadIdx.x & 15;
  const bool on = i < NT / kWave;
  const float m = on ? sm.m[i] : -INFINITY, c = on ? sm.c[i] : kRefFloor;
  const double s = on ? sm.s[i] : 0.0, w = on ? sm.w[i] : 0.0;
  RowTotals t;
  t.m = row16_max_all_f32(m);
  t.c = row16_max_all_f32(c);
  const float down = c - t.c;
  const double by = (double)exp2_fast(down);
  t.s = lane_f64(row16_sum_f64(s * by), 15);
  t.w = lane_f64(row16_sum_f64((w + (double)down * s) * by), 15);
  t.ahead = __builtin_amdgcn_readlane(wave_scan_i32(on ? sm.ahead[i] : 0), 15);
  return t;
}

// Sweep of vectors lo .. hi - 1 of a row by a workgroup of NT lanes; r keeps the lane's own part.  ONCE: read past the last-level cache.
template <int DT, int NT, bool ENT, bool TOP, bool ONCE>
__device__ __forceinline__ void sweep_vectors(const void* row, int V, int lo, int hi, float L, float zt, int token, RowSums& r) {
  constexpr int U = kAhead;
  const int whole = min(hi, V / Elem<DT>::per_vec), tid = threadIdx.x;
  r.init(L);
  int i0 = lo;
  for (; i0 + U * NT <= whole; i0 += U * NT) {         // (the same number of rounds in every lane)
    u32x4 q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) q[u] = ONCE ? load_vec_nt(row, i0 + u * NT + tid) : load_vec(row, i0 + u * NT + tid);
#pragma unroll
    for (int u = 0; u < U; ++u) add_vector<DT, ENT, TOP>(q[u], i0 + u * NT + tid, L, zt, token, r);
    r.flush();
  }
  if (i0 < hi) {                                       // the last, partial round
    u32x4 q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * NT + tid;
      q[u] = no_mass<DT>();
      if (i < whole) q[u] = ONCE ? load_vec_nt(row, i) : load_vec(row, i);
      else if (i < hi) q[u] = load_row_vec<DT>(row, V, i);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * NT < hi) add_vector<DT, ENT, TOP>(q[u], i0 + u * NT + tid, L, zt, token, r);
    r.flush();
  }
}
template <int DT, int NT, bool ENT, bool TOP>
__device__ __forceinline__ void sweep_row(const void* row, int V, int lo, int hi, bool once, float L, float zt, int token,
                                          RowSums& r) {
  if (once) sweep_vectors<DT, NT, ENT, TOP, true>(row, V, lo, hi, L, zt, token, r);
  else sweep_vectors<DT, NT, ENT, TOP, false>(row, V, lo, hi, L, zt, token, r);
}

// What a workgroup leaves of its part of a row that several sweep.
struct alignas(16) RowPart {
  double s, w;
  float m, c;
  int ahead;
  float zt;                          // the token's logit
};

// Totals of a row from its parts, in every lane: up to 64, one a lane.
__device__ __forceinline__ RowTotals fold_parts(const RowPart* parts, int n, float* zt) {
  const int lane = threadIdx.x & 63;
  RowPart p = {0.0, 0.0, -INFINITY, kRefFloor, 0, 0.f};
  if (lane < n) p = parts[lane];
  RowTotals t;
  t.m = wave_max_f32(p.m);
  t.c = wave_max_f32(p.c);
  const float down = p.c - t.c;
  const double by = (double)exp2_fast(down);
  t.s = wave_sum_f64(p.s * by);
  t.w = wave_sum_f64((p.w + (double)down * p.s) * by);
  t.ahead = __builtin_amdgcn_readlane(wave_scan_i32(p.ahead), kWave - 1);
  *zt = lane_f32(p.zt, 0);
  return t;
}

constexpr int kPartThreads = 256;
constexpr int kMaxRowParts = 64;        // one a lane
constexpr int kKeysAhead = 16;          // keys of a lane of the join at most

// How a row is divided: `n` parts of `vecs` vectors, the last one of what is left.  One part: one workgroup sweeps the row.
struct Split {
  int n, vecs;
  // lanes of a part that leave a key of their own: all while the join has registers for them, else one of each number
  __host__ __device__ int keys() const { return n <= kKeysAhead ? kPartThreads : kWave; }
};

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
  Split split;
  RowPart* parts;                    // [rows, split.n]
  uint64_t* keys;                    // [rows, split.n, split.keys()] the lanes' largest entries
  bool once;
  long long first;                   // position of the launch's first workgroup (whole rows)
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
  if ((int)threadIdx.x < a.n_top) {
    a.top_token[at * a.n_top + threadIdx.x] = -1;
    a.top_logprob[at * a.n_top + threadIdx.x] = bad ? x : -INFINITY;
  }
  if (threadIdx.x != 0) return;
  if (a.logprob) a.logprob[at] = x;
  if (a.lse) a.lse[at] = x;
  if (a.entropy) a.entropy[at] = x;
  if (a.rank) a.rank[at] = 0;
  if (a.flags) a.flags[at] = bad ? SV_FLAG_BAD_ROW : 0;
}

// The n first entries of a row in the order by value and, among equal ones, by token.  After the sweep every lane knows
// its largest entry, and the vector that holds it.  An entry among the n first lies in one of the n lanes that are first
// by (value, vector): any other lane has n entries before all of its own.  So
//  - a value that n lanes reach at least is found: of every wavefront its first few lanes, of those the n-th,
//  - the vectors of the lanes that reach it (n and a few more) are read again, the entries that reach it ranked by counting.
// The sweep pays two instructions a vector for this, whatever the row holds.  Where very many lanes reach the value
// (equal logits), the lanes are ranked first and n of them kept; lists that outgrow their places (rows of equal
// logits in many parts; large entries that all lie in few lanes) are walked n times instead, for one key each.
constexpr int kCandidates = 1024;
constexpr int kFewLanes = 128;

struct TopScratch {
  uint64_t lanes[kCandidates], first[SV_TOP_MAX], found[kCandidates], best[16];
  float value[kWave], low;
  int n_lanes, n_found;
};

// key(value, number): in descending order, equal values by ascending number; 0: no entry with mass.
__device__ __forceinline__ uint64_t key_of(float z, int number, float L) {
  return z * L >= kRefFloor ? (uint64_t)ordered(z) << 32 | (uint32_t)~number : 0;
}
__device__ __forceinline__ float value_of(uint64_t key) { return key ? from_ordered((uint32_t)(key >> 32)) : -INFINITY; }
__device__ __forceinline__ int number_of(uint64_t key) { return (int)~(uint32_t)key; }

// Largest key of the workgroup.
template <int NT>
__device__ __forceinline__ uint64_t block_max_u64(uint64_t key, uint64_t* sm) {
  key = wave_max_u64(key);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = key;
  __syncthreads();
  for (int w = 0; w < NT / kWave; ++w) key = sm[w] > key ? sm[w] : key;
  return key;
}

// Every key of a list of n distinct ones with its rank, by lanes tid, tid + step, ...: take(rank, key).
template <class Take>
__device__ __forceinline__ void rank_keys(const uint64_t* keys, int n, int tid, int step, Take&& take) {
  for (int t = tid; t < n; t += step) {
    const uint64_t key = keys[t];
    int rank = 0;
    for (int m = 0; m < n; ++m) rank += keys[m] > key;
    take(rank, key);
  }
}

// NT lanes; each has the keys (value, vector) of K lanes of the sweep (0: none); a lane of the sweep had the vectors that
// are `lanes` apart in its part of the row.  What the first wavefront alone can do, it does, emit() among it: with many
// rows to a compute unit the instructions of all wavefronts count (4096 x 8000 bf16 with 20 alternatives: 46 us with the
// ranks formed by all of them, 36 so).
// The second wavefront does what `meanwhile` says while the first one looks for the value.
template <int DT, int NT, int K, class Meanwhile, class Emit>
__device__ __forceinline__ void alternatives(const void* row, int V, float L, int n, Split split, int lanes_apart,
                                             const uint64_t (&keys)[K], TopScratch& sm, Meanwhile&& meanwhile, Emit&& emit) {
  constexpr int EPV = Elem<DT>::per_vec, kWaves = NT / kWave;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n_vec = vectors_of<DT>(V);
  auto each_lane_key = [&](auto&& f) {
#pragma unroll
    for (int j = 0; j < K; ++j) f(keys[j]);
  };
  uint64_t best = 0;
  each_lane_key([&](uint64_t k) { best = k > best ? k : best; });
  // the first few values of every wavefront; n of them in all, at least
  const int few = min(min(n, (n + kWaves - 1) / kWaves + 2), kWave / kWaves), n_values = few * kWaves;
  float left = value_of(best);
  for (int j = 0; j < few; ++j) {
    const float v = wave_max_f32(left);
    if (lane == __builtin_ctzll(__ballot(left == v))) {
      left = -INFINITY;
      sm.value[wave * few + j] = v;
    }
  }
  if (tid == 0) sm.n_lanes = sm.n_found = 0;
  __syncthreads();
  if (wave == 0) {
    const float mine = lane < n_values ? sm.value[lane] : -INFINITY;
    int before = 0;
    for (int l = 0; l < n_values; ++l) {
      const float v = sm.value[l];
      before += v > mine || (v == mine && l < lane);
    }
    if (lane < n_values && before == n - 1) sm.low = mine;
  } else if (wave == 1) {
    meanwhile();
  }
  __syncthreads();
  const float low = sm.low;
  each_lane_key([&](uint64_t key) {
    if (key == 0 || value_of(key) < low) return;
    const int at = atomicAdd(&sm.n_lanes, 1);
    if (at < kCandidates) sm.lanes[at] = key;
  });
  __syncthreads();
  int n_lanes = sm.n_lanes;
  const uint64_t* lanes = sm.lanes;
  float last_z = low;                                  // entries before (value, vector) are looked at
  int last_vec = V;
  if (n_lanes > kFewLanes) {
    if (n_lanes <= kCandidates) {
      rank_keys(sm.lanes, n_lanes, tid, NT, [&](int rank, uint64_t key) { if (rank < n) sm.first[rank] = key; });
    } else {
      uint64_t before = ~0ull;
      for (int r = 0; r < n; ++r) {
        uint64_t key = 0;
        each_lane_key([&](uint64_t k) { key = k < before && k > key ? k : key; });
        before = block_max_u64<NT>(key, sm.best);
        if (tid == 0) sm.first[r] = before;
      }
    }
    __syncthreads();
    lanes = sm.first;
    n_lanes = n;
    last_vec = number_of(sm.first[n - 1]);
    last_z = value_of(sm.first[n - 1]);
  }
  const int per_lane = split.vecs / lanes_apart;
  auto visit = [&](auto&& take) {                      // (kAhead vectors of a lane under way: a trip to memory for most rows)
    const int n_visits = n_lanes * per_lane;
    for (int p0 = tid; p0 < n_visits; p0 += kAhead * NT) {
      u32x4 q[kAhead];
      int number[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int p = p0 + u * NT;
        number[u] = n_vec;
        q[u] = no_mass<DT>();
        if (p >= n_visits) continue;
        const int e = (int)((uint32_t)p / (uint32_t)n_lanes), of = number_of(lanes[p - e * n_lanes]);
        const int part = split.n == 1 ? 0 : (int)((uint32_t)of / (uint32_t)split.vecs) * split.vecs;
        number[u] = part + (int)((uint32_t)(of - part) % (uint32_t)lanes_apart) + e * lanes_apart;
        if (number[u] < n_vec) q[u] = load_row_vec<DT>(row, V, number[u]);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (number[u] >= n_vec) continue;
        float f[EPV];
        unpack<DT>(q[u], f);
#pragma unroll
        for (int j = 0; j < EPV; ++j) {
          if (!(f[j] >= last_z)) continue;
          const uint64_t key = key_of(f[j], number[u] * EPV + j, L);
          if (key && (f[j] > last_z || number[u] <= last_vec)) take(key);
        }
      }
    }
  };
  visit([&](uint64_t key) {
    const int at = atomicAdd(&sm.n_found, 1);
    if (at < kCandidates) sm.found[at] = key;
  });
  __syncthreads();
  const int n_found = sm.n_found;
  if (n_found <= kCandidates) {
    if (wave != 0) return;
    rank_keys(sm.found, n_found, lane, kWave, [&](int rank, uint64_t key) { if (rank < n) emit(rank, key); });
    if (lane < n && lane >= n_found) emit(lane, 0);
    return;
  }
  uint64_t before = ~0ull;
  for (int r = 0; r < n; ++r) {
    uint64_t key = 0;
    visit([&](uint64_t k) { key = k < before && k > key ? k : key; });
    before = block_max_u64<NT>(key, sm.best);
    if (tid == 0) emit(r, before);
  }
}

// The row of a position: its address, or none because nothing is asked for or nothing is there (blank), or bad.
struct Position {
  const void* row;
  int token;
  bool bad;
};
template <int DT>
__device__ __forceinline__ Position locate(const ScoreArgs& a, long long at) {
  Position p = {nullptr, -1, false};
  if (a.tokens) {
    p.token = a.tokens[at];
    if (p.token == -1) return p;
  }
  if (a.offsets) {
    const int b = (int)(at / a.P), i = (int)(at % a.P);
    const long long lo = a.offsets[b], hi = a.offsets[b + 1];
    if (i >= hi - lo) return p;
    at = lo + i;
    if (at < 0 || at >= a.n_rows) { p.bad = true; return p; }
  }
  p.row = static_cast<const char*>(a.z) + (size_t)at * (size_t)a.stride * Elem<DT>::bytes;
  return p;
}
template <int DT>
__device__ __forceinline__ float token_logit(const void* row, int token, int V) {
  return token >= 0 && token < V ? load_elem<DT>(row, token) : __builtin_nanf("");
}

// Results of a row that is there.  totals(&zt) are asked for by one wavefront, after the barrier that follows what it needs.
template <int DT, int NT, bool TOP, int K, class Totals>
__device__ __forceinline__ void write_row(const ScoreArgs& a, long long at, const Position& p, Totals&& totals,
                                          const uint64_t (&keys)[K], int lanes_apart) {
  __shared__ double row_lse;                           // NaN: a bad row
  auto logprob_of = [&](float z, double lse) {
    return lse != lse ? __builtin_nanf("") : z * a.sc.L < kRefFloor ? -INFINITY : (float)((double)z * a.sc.inv_t - lse);
  };
  auto write_totals = [&] {
    float zt;
    const RowTotals t = totals(&zt);
    const bool bad = t.bad(), given = p.token >= 0 && p.token < a.V;
    const double lse = bad ? __builtin_nan("") : t.lse(a.sc);
    if ((threadIdx.x & 63) != 0) return;
    row_lse = lse;
    if (a.logprob) a.logprob[at] = given ? logprob_of(zt, lse) : __builtin_nanf("");
    if (a.lse) a.lse[at] = (float)lse;
    if (a.entropy) a.entropy[at] = bad ? __builtin_nanf("") : (float)t.entropy();
    if (a.rank) a.rank[at] = given && !bad ? 1 + t.ahead : 0;
    if (a.flags) a.flags[at] = bad ? SV_FLAG_BAD_ROW : a.tokens && !given ? SV_FLAG_BAD_TOKEN : 0;
  };
  if constexpr (TOP) {
    __shared__ TopScratch top;
    alternatives<DT, NT>(p.row, a.V, a.sc.L, a.n_top, a.split, lanes_apart, keys, top, write_totals,
                         [&](int rank, uint64_t key) {
                           const double lse = row_lse;
                           a.top_token[at * a.n_top + rank] = key && lse == lse ? number_of(key) : -1;
                           a.top_logprob[at * a.n_top + rank] = logprob_of(value_of(key), lse);
                         });
  } else if (threadIdx.x < kWave) {
    write_totals();
  }
}

// One workgroup to a row: 4096 x 128256 bf16, rank, entropy and one alternative, 179 us = 5.9 TB/s, bound by HBM (its ten issue
// slots an entry would allow 7.9).
template <int DT, int NT, bool ENT, bool TOP>
__global__ __launch_bounds__(NT, 8) void token_logprobs_kernel(const ScoreArgs a) {
  __shared__ RowScratch sm;
  const long long at = a.first + blockIdx.x;
  const Position p = locate<DT>(a, at);
  if (!p.row) return write_blank(a, at, p.bad);
  const float zt = token_logit<DT>(p.row, p.token, a.V);
  RowSums r;
  sweep_row<DT, NT, ENT, TOP>(p.row, a.V, 0, vectors_of<DT>(a.V), a.once, a.sc.L, zt, p.token, r);
  leave_row(r, sm);
  if (!TOP) __syncthreads();                           // (with alternatives they have the barrier)
  const uint64_t best[1] = {key_of(r.m, r.best, a.sc.L)};
  write_row<DT, NT, TOP>(a, at, p, [&](float* z) { *z = zt; return fold_row<NT>(sm); }, best, NT);
}

// Several workgroups to a row: first its parts, then one workgroup a row for the results.  A compute unit needs 10 us for the
// instructions of 152064 bf16 entries and longer for their loads one round after the other, so one row takes 14 us this way and 31 with a
// workgroup (entropy, rank, 20 alternatives; 9 and 26 without these); 316 rows 40 and 48 us, bound by the start and the end of each launch
// and the rest by HBM.
template <int DT, bool ENT, bool TOP>
__global__ __launch_bounds__(kPartThreads, 8) void token_logprobs_part_kernel(const ScoreArgs a) {
  __shared__ RowScratch sm;
  const long long at = blockIdx.x / a.split.n;
  const int part = blockIdx.x % a.split.n;
  const Position p = locate<DT>(a, at);
  if (!p.row) return;
  const float zt = token_logit<DT>(p.row, p.token, a.V);
  RowSums r;
  const int lo = part * a.split.vecs, hi = min(lo + a.split.vecs, vectors_of<DT>(a.V));
  sweep_row<DT, kPartThreads, ENT, TOP>(p.row, a.V, lo, hi, a.once, a.sc.L, zt, p.token, r);
  leave_row(r, sm);
  __shared__ uint64_t best[TOP ? kPartThreads : 1];
  if (TOP) best[threadIdx.x] = key_of(r.m, r.best, a.sc.L);
  if (TOP && a.split.keys() == kPartThreads) a.keys[(size_t)blockIdx.x * kPartThreads + threadIdx.x] = best[threadIdx.x];
  __syncthreads();
  if (threadIdx.x >= kWave) return;
  if (TOP && a.split.keys() == kWave) {
    uint64_t key = best[threadIdx.x];
#pragma unroll
    for (int w = 1; w < kPartThreads / kWave; ++w) key = best[w * kWave + threadIdx.x] > key ? best[w * kWave + threadIdx.x] : key;
    a.keys[(size_t)blockIdx.x * kWave + threadIdx.x] = key;
  }
  const RowTotals t = fold_row<kPartThreads>(sm);
  if (threadIdx.x == 0) a.parts[blockIdx.x] = {t.s, t.w, t.m, t.c, t.ahead, zt};
}

template <int DT, bool TOP>
__global__ __launch_bounds__(kPartThreads) void token_logprobs_join_kernel(const ScoreArgs a) {
  static_assert(kKeysAhead * kPartThreads >= kMaxRowParts * kWave, "keys of a row");
  const long long at = blockIdx.x;
  uint64_t keys[TOP ? kKeysAhead : 1] = {};
  if (TOP) {                                           // (asked for before it is known whether the row is there)
    const int n = a.split.n * a.split.keys();
#pragma unroll
    for (int j = 0; j < kKeysAhead; ++j) {
      const int i = j * kPartThreads + threadIdx.x;
      if (i < n) keys[TOP ? j : 0] = a.keys[(size_t)at * n + i];
    }
  }
  const Position p = locate<DT>(a, at);
  if (!p.row) return write_blank(a, at, p.bad);
  write_row<DT, kPartThreads, TOP>(a, at, p, [&](float* z) { return fold_parts(a.parts + at * a.split.n, a.split.n, z); },
                                   keys, a.split.keys());
}

inline int round_up(int n, int to) { return (n + to - 1) / to * to; }

// A call with few rows of many rounds of loads divides each into parts of whole rounds, as many as give the chip its places for
// workgroups.  One workgroup to a row / divided, us, with entropy and rank:
//  by rounds: without alternatives 6, 10 and 16 rounds of bf16, 1 row 10.7/8.6, 15.0/8.8, 23.2/8.5; 144 rows 12.3/12.2, 17.9/14.2, 26.4/17.6;
//    f32, 1 row 7.3/8.6, 9.9/8.5, 14.9/8.2; 144 rows 9.9/10.5, 13.5/12.1, 19.6/14.4.  With 20, whose join is longer, bf16, 1 row 14.1/13.5,
//    18.6/13.7, 26.8/13.9; 144 rows 16.7/18.5, 21.5/21.4, 30.9/25.7; f32, 1 row 10.9/12.2, 13.4/12.5, 18.9/12.5; 144 rows 13.1/16.5, 17.1/18.6,
//    23.4/21.9.  Ten rounds is where calls with alternatives meet; those without meet at six to eight, and lose up to 6 us by one line for both.
//  by rows, without / with 20 alternatives: bf16 x 152064, 256 rows 31.2/27.1, 36.1/34.5; 682 rows 51.4/50.8, 63.9/63.0; 1024 rows 66.8/69.4,
//    79.7/87.4.  f32 x 152064, 256 rows 40.2/31.7, 50.1/41.0; 682 rows 68.7/74.9, 83.2/91.1.  bf16 x 80000, 256 rows 19.1/19.0, 23.3/26.1; 682
//    rows 31.1/34.4, 37.6/41.5.  f32 x 40000, 144 rows 13.8/12.2, 17.4/18.7; 256 rows 14.7/15.6, 18.7/22.4; 682 rows 24.3/28.4, 29.6/36.3.
//    682 is where long bf16 rows meet; shorter and f32 ones meet at 150 to 400 and lose up to a quarter between there and the line.
//  gradient, by rows (divided, it reads the logits twice): bf16 x 152064, 64 rows 25.7/18.2, 96 rows 26.3/24.1, 128 rows 26.8/28.6, 192 rows
//    28.4/40.2.  f32 x 152064, 96 rows 37.3/34.9, 128 rows 42.6/46.0.  bf16 x 80000, 96 rows 17.6/17.1, 128 rows 17.7/19.2.  f32 x 40000, 64 rows
//    12.6/12.2, 96 rows 12.9/14.5, 192 rows 14.7/21.6.
constexpr int kPlaces = 4096, kFewRounds = 10, kScoreRows = 682, kGradRows = 96;
inline Split whole_row(int V, int dtype) {
  const int per_vec = 16 / elem_bytes(dtype);
  return {1, (V + per_vec - 1) / per_vec};
}
inline Split split_of(long long rows, int V, int dtype, int max_rows) {
  const Split whole = whole_row(V, dtype);
  constexpr int kRound = kPartThreads * kAhead;
  const int rounds = (whole.vecs + kRound - 1) / kRound;
  if (rows < 1 || rows > max_rows || rounds < kFewRounds) return whole;
  const int n = (int)min((kPlaces + rows - 1) / rows, (long long)min(rounds, kMaxRowParts));
  const int vecs = (rounds + n - 1) / n * kRound;
  return {(whole.vecs + vecs - 1) / vecs, vecs};
}

template <int DT, bool ENT>
void launch_score(ScoreArgs a, long long rows, hipStream_t st) {
  if (a.split.n > 1) {                                 // (few rows)
    const dim3 grid((unsigned)rows), parts((unsigned)(rows * a.split.n)), block(kPartThreads);
    if (a.n_top > 0) {
      hipLaunchKernelGGL((token_logprobs_part_kernel<DT, ENT, true>), parts, block, 0, st, a);
      hipLaunchKernelGGL((token_logprobs_join_kernel<DT, true>), grid, block, 0, st, a);
    } else {
      hipLaunchKernelGGL((token_logprobs_part_kernel<DT, ENT, false>), parts, block, 0, st, a);
      hipLaunchKernelGGL((token_logprobs_join_kernel<DT, false>), grid, block, 0, st, a);
    }
    return;
  }
  auto go = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    a.split.vecs = round_up(a.split.vecs, NT);
    in_launches(rows, NT, [&](long long first, dim3 grid) {
      a.first = first;
      if (a.n_top > 0) hipLaunchKernelGGL((token_logprobs_kernel<DT, NT, ENT, true>), grid, dim3(NT), 0, st, a);
      else hipLaunchKernelGGL((token_logprobs_kernel<DT, NT, ENT, false>), grid, dim3(NT), 0, st, a);
    });
  };
  // many short rows: small workgroups, whose ends overlap other rows' sweeps (4096 x 8000 bf16, 20 alternatives: 36 us, 48 with
  // 512 lanes); few rows: more lanes to each (144 x 32000: 13 us, 17 with 256)
  if (rows >= 1024 && a.split.vecs <= 4096) go(std::integral_constant<int, 256>());
  else go(std::integral_constant<int, 512>());
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
  Split split;
  RowPart* parts;                    // [rows, split.n]
  long long first;                   // row of the launch's first workgroup (whole rows)
};

__device__ __forceinline__ u32x4 load_bytes(const char* row, uint32_t at) {
  return __builtin_nontemporal_load(reinterpret_cast<const u32x4_row*>(row + at));
}
template <int DT>
__device__ __forceinline__ u32x4 pack_vec(const float (&f)[Elem<DT>::per_vec]) {
  if constexpr (DT == DT_F32)
    return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  else
    return u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
}
// Vector i of a row of V entries, the counterpart of load_row_vec.
template <int DT>
__device__ __forceinline__ void store_row_vec(void* row, int V, int i, const float (&f)[Elem<DT>::per_vec]) {
  constexpr int EPV = Elem<DT>::per_vec;
  const u32x4 q = pack_vec<DT>(f);
  if (i < V / EPV) {
    __builtin_nontemporal_store(q, reinterpret_cast<u32x4_row*>(row) + i);
    return;
  }
  for (int j = 0; j < V - i * EPV; ++j) {
    if constexpr (DT == DT_F32) reinterpret_cast<uint32_t*>(row)[i * EPV + j] = q[j];
    else reinterpret_cast<uint16_t*>(row)[i * EPV + j] = (uint16_t)(q[j >> 1] >> (16 * (j & 1)));
  }
}

// dz_v = 2^y (a0 + a1 y), and g / T more at the token:  log p = (y - log2 S) ln 2.
struct RowGrad {
  float c, a0, a1, at_token;
};

// A row's gradient in these terms; its log-probability, entropy and flags by the lane that `writes`.
template <bool ENT>
__device__ __forceinline__ RowGrad row_grad(const GradArgs& a, long long at, int token, float zt, const RowTotals& t,
                                            bool writes) {
  const bool given = token >= 0 && token < a.V, bad = t.bad();
  if (writes) {
    const double lp = zt * a.sc.L < kRefFloor ? -INFINITY : (double)zt * a.sc.inv_t - t.lse(a.sc);
    if (a.logprob) a.logprob[at] = bad || !given ? __builtin_nanf("") : (float)lp;
    if (a.entropy) a.entropy[at] = bad ? __builtin_nanf("") : (float)t.entropy();
    if (a.flags) a.flags[at] = (bad ? SV_FLAG_BAD_ROW : 0) | (given ? 0 : SV_FLAG_BAD_TOKEN);
  }
  const float nan = __builtin_nanf("");
  if (bad || !given) return {0.f, nan, nan, nan};
  const double g = (double)a.g_logprob[at], h = ENT && a.g_entropy ? (double)a.g_entropy[at] : 0.0;
  const double inv_s = a.sc.inv_t / t.s;
  return {t.c, (float)(-inv_s * (g + h * (ENT ? t.entropy() - t.log2_s() * kLn2 : 0.0))), (float)(-inv_s * h * kLn2),
          (float)(g * a.sc.inv_t)};
}

// Gradient of vector i, in place of its logits.
template <int DT, bool ENT>
__device__ __forceinline__ void grad_of(float (&f)[Elem<DT>::per_vec], int i, float L, int token, const RowGrad& r) {
  constexpr int EPV = Elem<DT>::per_vec;
#pragma unroll
  for (int j = 0; j < EPV; ++j) {
    const float y = __builtin_fmaf(f[j], L, -r.c);
    f[j] = exp2_fast(y) * (ENT ? __builtin_fmaf(fmaxf(y, kLowY), r.a1, r.a0) : r.a0);
  }
  if (token / EPV == i) {
#pragma unroll
    for (int j = 0; j < EPV; ++j) f[j] += token % EPV == j ? r.at_token : 0.f;
  }
}
template <int DT, bool ENT>
__device__ __forceinline__ void store_grad(void* out, int i, const u32x4& q, float L, int token, const RowGrad& r) {
  float f[Elem<DT>::per_vec];
  unpack<DT>(q, f);
  grad_of<DT, ENT>(f, i, L, token, r);
  __builtin_nontemporal_store(pack_vec<DT>(f), reinterpret_cast<u32x4_row*>(static_cast<char*>(out) + i * 16u));
}

// Vectors lo .. hi - 1 of a row without a token (zeros) or of a bad one (NaN).
template <int DT, int NT>
__device__ __forceinline__ void fill_row(void* out, int V, int lo, int hi, float x) {
  constexpr int EPV = Elem<DT>::per_vec;
  float f[EPV];
#pragma unroll
  for (int j = 0; j < EPV; ++j) f[j] = x;
  for (int i = lo + threadIdx.x; i < hi; i += NT) store_row_vec<DT>(out, V, i, f);
}
__device__ __forceinline__ void write_no_token(const GradArgs& a, long long at) {
  if (a.logprob) a.logprob[at] = 0.f;
  if (a.entropy) a.entropy[at] = 0.f;
  if (a.flags) a.flags[at] = 0;
}

template <int DT, int NT, bool ENT>
__device__ __forceinline__ void store_grads(const void* row, void* out, int V, int lo, int hi, float L, int token,
                                            const RowGrad& r) {
  if (r.a0 != r.a0) return fill_row<DT, NT>(out, V, lo, hi, r.a0);
  const int whole = min(hi, V / Elem<DT>::per_vec);
  int i = lo + threadIdx.x;
  for (; i + (kAhead - 1) * NT < whole; i += kAhead * NT) {
    u32x4 q[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) q[u] = load_vec(row, i + u * NT);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) store_grad<DT, ENT>(out, i + u * NT, q[u], L, token, r);
  }
  for (; i < hi; i += NT) {
    float f[Elem<DT>::per_vec];
    unpack<DT>(load_row_vec<DT>(row, V, i), f);
    grad_of<DT, ENT>(f, i, L, token, r);
    store_row_vec<DT>(out, V, i, f);
  }
}

// One workgroup to a row.  The first R vectors of every lane stay in its registers from the sums to the gradient; the
// others are read again.  2048 x 152064 bf16 with entropy: 235 us, 5.0 TB/s of logits read and gradients written (292 us with the
// logits read twice); 4096 x 32000 f32: 178 us, 5.9 TB/s.  Both past the last-level cache: 264 and 197 us through it.
template <int DT, int NT, int R, int WAVES, bool ENT>
__global__ __launch_bounds__(NT, WAVES) void token_logprobs_grad_kernel(const GradArgs a) {
  __shared__ RowScratch sm;
  const long long at = a.first + blockIdx.x;
  const int V = a.V, token = a.tokens[at], n_vec = vectors_of<DT>(V), whole = V / Elem<DT>::per_vec, tid = threadIdx.x;
  const char* row = static_cast<const char*>(a.z) + (size_t)at * (size_t)a.stride * Elem<DT>::bytes;
  char* out = static_cast<char*>(a.dz) + (size_t)at * (size_t)a.dz_stride * Elem<DT>::bytes;
  if (token == -1) {
    fill_row<DT, NT>(out, V, 0, n_vec, 0.f);
    if (tid == 0) write_no_token(a, at);
    return;
  }
  // The lane's number, each time anew: what is formed from it for a load is not kept for the store.
  auto lane = [&] {
    int l = tid;
    asm volatile("" : "+v"(l));
    return l;
  };
  u32x4 q[R];
#pragma unroll
  for (int u = 0; u < R; ++u) {                        // (uniform base, 32-bit offset: one register of address)
    if (u * NT >= whole) continue;
    q[u] = load_bytes(row, min(u * NT + lane(), whole - 1) * 16u);
  }
  const float zt = token_logit<DT>(row, token, V);      // (before anything is written: dz may be z)
  RowSums r;
  r.init(a.sc.L);
#pragma unroll
  for (int u = 0; u < R; ++u) {
    if (u * NT < whole)
      add_vector<DT, ENT, false>(u * NT + lane() < whole ? q[u] : no_mass<DT>(), 0, a.sc.L, __builtin_nanf(""), -1, r);
    if (u % kAhead == kAhead - 1) r.flush();
    __builtin_amdgcn_sched_barrier(0);                 // (vector after vector: unpacked ahead they take the registers)
  }
  r.flush();
  const int rest = min(R * NT, whole);                 // past the registers, and past the last whole vector
#pragma unroll 1
  for (int i0 = rest; i0 < n_vec; i0 += NT) {
    const int i = i0 + tid;
    const u32x4 v = i < n_vec ? load_row_vec<DT>(row, V, i) : no_mass<DT>();
    add_vector<DT, ENT, false>(v, 0, a.sc.L, __builtin_nanf(""), -1, r);
    r.flush();
  }
  leave_row(r, sm);
  __syncthreads();
  const RowGrad d = row_grad<ENT>(a, at, token, zt, fold_row<NT>(sm), tid == 0);
  if (d.a0 != d.a0) return fill_row<DT, NT>(out, V, 0, n_vec, d.a0);
#pragma unroll
  for (int u = 0; u < R; ++u) {
    const int i = u * NT + lane();
    if (i < whole) store_grad<DT, ENT>(out, i, q[u], a.sc.L, token, d);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (rest < n_vec) store_grads<DT, NT, ENT>(row, out, V, rest, n_vec, a.sc.L, token, d);
}

// Several workgroups to a row, after token_logprobs_part_kernel has left the parts' sums.
template <int DT, bool ENT>
__global__ __launch_bounds__(kPartThreads) void token_logprobs_grad_part_kernel(const GradArgs a) {
  const long long at = blockIdx.x / a.split.n;
  const int part = blockIdx.x % a.split.n, V = a.V, token = a.tokens[at];
  const int lo = part * a.split.vecs, hi = min(lo + a.split.vecs, vectors_of<DT>(V));
  const void* row = static_cast<const char*>(a.z) + (size_t)at * (size_t)a.stride * Elem<DT>::bytes;
  char* out = static_cast<char*>(a.dz) + (size_t)at * (size_t)a.dz_stride * Elem<DT>::bytes;
  const bool writes = part == 0 && threadIdx.x == 0;
  if (token == -1) {
    fill_row<DT, kPartThreads>(out, V, lo, hi, 0.f);
    if (writes) write_no_token(a, at);
    return;
  }
  float zt;
  const RowTotals t = fold_parts(a.parts + at * a.split.n, a.split.n, &zt);
  const RowGrad d = row_grad<ENT>(a, at, token, zt, t, writes);
  store_grads<DT, kPartThreads, ENT>(row, out, V, lo, hi, a.sc.L, token, d);
}

template <int DT, bool ENT>
void launch_grad(GradArgs a, int rows, hipStream_t st) {
  if (a.split.n > 1) {
    ScoreArgs s = {};
    s.z = a.z; s.stride = a.stride; s.tokens = a.tokens; s.P = 1; s.V = a.V; s.sc = a.sc; s.split = a.split; s.parts = a.parts;
    const dim3 grid((unsigned)((long long)rows * a.split.n)), block(kPartThreads);
    hipLaunchKernelGGL((token_logprobs_part_kernel<DT, ENT, false>), grid, block, 0, st, s);
    hipLaunchKernelGGL((token_logprobs_grad_part_kernel<DT, ENT>), grid, block, 0, st, a);
    return;
  }
  const int n_vec = (a.V + Elem<DT>::per_vec - 1) / Elem<DT>::per_vec;
  auto go = [&](auto kernel, int lanes) {
    in_launches(rows, lanes, [&](long long first, dim3 grid) {
      a.first = first;
      hipLaunchKernelGGL(kernel, grid, dim3(lanes), 0, st, a);
    });
  };
  // lanes and registers by the row's length, so that a short row leaves the compute unit room for others
  if (n_vec <= 256 * 8) go(token_logprobs_grad_kernel<DT, 256, 8, 6, ENT>, 256);
  else if (n_vec <= 512 * 8) go(token_logprobs_grad_kernel<DT, 512, 8, 6, ENT>, 512);
  else if (n_vec <= 512 * 16) go(token_logprobs_grad_kernel<DT, 512, 12, 5, ENT>, 512);
  else go(token_logprobs_grad_kernel<DT, 1024, 19, 4, ENT>, 1024);
}

// Parts and, with alternatives, the lanes' keys of the rows that are divided.
inline size_t parts_bytes(long long rows, const Split& s) { return ws_round((size_t)rows * s.n * sizeof(RowPart)); }
inline size_t keys_bytes(long long rows, const Split& s) { return ws_round((size_t)rows * s.n * s.keys() * 8); }
inline size_t score_bytes(long long rows, int V, int dtype, int n_top) {
  const Split s = split_of(rows, V, dtype, kScoreRows);
  return s.n == 1 ? 0 : parts_bytes(rows, s) + (n_top > 0 ? keys_bytes(rows, s) : 0);
}

}  // namespace sv

extern "C" size_t sv_token_logprobs_workspace_bytes(int64_t rows, int V, int dtype, int n_top) {
  if (rows < 0 || rows > 0x7fffffffLL || V < 1 || V > (1 << 24) || sv::elem_bytes(dtype) == 0 || n_top < 0 || n_top > SV_TOP_MAX)
    return 0;
  return sv::score_bytes(rows, V, dtype, n_top);
}

extern "C" int sv_token_logprobs(const void* z, int64_t z_stride, const int32_t* t_offsets_or_null, int n_rows,
                                 const int32_t* tokens_or_null, int B, int P, int V, int dtype, float temperature,
                                 int n_top, float* logprob_or_null, float* lse_or_null, float* entropy_or_null,
                                 int32_t* rank_or_null, int32_t* top_token_or_null, float* top_logprob_or_null,
                                 uint32_t* flags_or_null, void* ws_or_null, size_t ws_bytes, sv_stream_t stream) {
  using namespace sv;
  SV_REQUIRE(dtype == SV_F32 || dtype == SV_BF16, SV_ERR_DTYPE);
  SV_REQUIRE(B >= 0 && P >= 1 && V >= 1 && z_stride >= V && n_top >= 0, SV_ERR_INVALID_ARG);
  SV_REQUIRE(!t_offsets_or_null || n_rows >= 0, SV_ERR_INVALID_ARG);
  ScoreArgs a = {};
  SV_REQUIRE(scale_of(temperature, &a.sc), SV_ERR_INVALID_ARG);
  SV_REQUIRE(V <= (1 << 24) && n_top <= SV_TOP_MAX && (long long)B * P <= 0x7fffffffLL, SV_ERR_TOO_LARGE);
  if (B == 0) return SV_OK;
  SV_REQUIRE(z || (t_offsets_or_null && n_rows == 0), SV_ERR_NULL);      // (no row: torch gives NULL as its address)
  SV_REQUIRE(tokens_or_null || (!logprob_or_null && !rank_or_null), SV_ERR_NULL);
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
  // 1024 x 152064 f32: 100 us past the last-level cache, 112 us through it; 144 x 32000 bf16: 14.3 and 12.5
  a.once = rows * V * elem_bytes(dtype) > kCacheBytes;
  a.split = ws_or_null ? split_of(rows, V, dtype, kScoreRows) : whole_row(V, dtype);
  if (ws_or_null) {
    SV_REQUIRE(is_aligned(ws_or_null, kWsAlign) && ws_bytes >= score_bytes(rows, V, dtype, n_top), SV_ERR_WORKSPACE);
    a.parts = static_cast<RowPart*>(ws_or_null);
    a.keys = reinterpret_cast<uint64_t*>(static_cast<char*>(ws_or_null) + parts_bytes(rows, a.split));
  }
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
                                      void* dz, int64_t dz_stride, uint32_t* flags_or_null, void* ws_or_null,
                                      size_t ws_bytes, sv_stream_t stream) {
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
  a.split = ws_or_null ? split_of(rows, V, dtype, kGradRows) : whole_row(V, dtype);
  if (ws_or_null) {
    SV_REQUIRE(is_aligned(ws_or_null, kWsAlign) && ws_bytes >= score_bytes(rows, V, dtype, 0), SV_ERR_WORKSPACE);
    a.parts = static_cast<RowPart*>(ws_or_null);
  }
  hipStream_t st = as_stream(stream);
  if (dtype == SV_F32) {
    if (ent) launch_grad<DT_F32, true>(a, rows, st);
    else launch_grad<DT_F32, false>(a, rows, st);
  } else {
    if (ent) launch_grad<DT_BF16, true>(a, rows, st);
    else launch_grad<DT_BF16, false>(a, rows, st);
  }
  return launch_status();
}
