// sv_embedding: scaled rows of a table.  sv_embedding_grad: the gradient of that table.
//
// The gradient sorts the tokens (least significant digit first, kDigitBits bits a pass, stable) and sums the rows of
// equal tokens in the order of their positions: no atomics on the result, the same bits from every call.
// Few tokens need no sort: one launch finds, orders and sums them.
// Positions whose id is no row sort behind all others.  The sort occupies a few workgroups for some
// microseconds a launch; the other workgroups of its launches write the table's zeros meanwhile.
#include <algorithm>

#include "sv_device.hpp"
#include "sv_host.hpp"

namespace sv {

constexpr int kChunkCols = 8;           // columns of one lane: 16 bytes of bfloat16, 32 of float32
constexpr int kEmbThreads = 256;
constexpr int kMinLanes = 8;            // lanes of a row at least

// The eight columns of chunk c of a row of D: 8c .. 8c + 7, or the row's last eight, of which the first `skip` are the chunk's
// before.  (A row of fewer than eight has its own, one by one.)
struct Columns {
  int at, skip;
};
__device__ __forceinline__ Columns columns_of(int D, int c) {
  const int at = max(min(c * kChunkCols, D - kChunkCols), 0);
  return {at, c * kChunkCols - at};
}
template <int DT>
struct Chunk {
  static constexpr int kVecs = kChunkCols / Elem<DT>::per_vec;
  u32x4 q[kVecs];
  template <bool ONCE = false>
  __device__ __forceinline__ void load(const void* row, int D, int c) {
    const char* p = static_cast<const char*>(row) + (size_t)columns_of(D, c).at * Elem<DT>::bytes;
    if (D >= kChunkCols) {
#pragma unroll
      for (int k = 0; k < kVecs; ++k) q[k] = ONCE ? load_vec_nt(p, k) : load_vec(p, k);
      return;
    }
#pragma unroll
    for (int k = 0; k < kVecs; ++k) q[k] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < kChunkCols; ++j) {
      if (j >= D) continue;
      if constexpr (DT == DT_F32) q[j / 4][j % 4] = reinterpret_cast<const uint32_t*>(p)[j];
      else q[0][j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[j] << (16 * (j & 1));
    }
  }
  __device__ __forceinline__ void get(float (&f)[kChunkCols]) const {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      float v[Elem<DT>::per_vec];
      unpack<DT>(q[k], v);
#pragma unroll
      for (int j = 0; j < Elem<DT>::per_vec; ++j) f[k * Elem<DT>::per_vec + j] = v[j];
    }
  }
  __device__ __forceinline__ void add_to(float (&sum)[kChunkCols]) const {
    float f[kChunkCols];
    get(f);
#pragma unroll
    for (int j = 0; j < kChunkCols; ++j) sum[j] += f[j];
  }
};

__device__ __forceinline__ void store_nt(void* row, int i, const u32x4& q) {      // not read again soon
  __builtin_nontemporal_store(q, reinterpret_cast<u32x4_row*>(row) + i);
}
// ONCE: the results are more than the last-level cache keeps for a later reader, and are written past it.
template <int DT, bool ONCE = true>
__device__ __forceinline__ void store_chunk(void* row, int D, int c, const float (&f)[kChunkCols]) {
  const Columns w = columns_of(D, c);
  char* p = static_cast<char*>(row) + (size_t)w.at * Elem<DT>::bytes;
  u32x4 q[2];
  if constexpr (DT == DT_F32) {
#pragma unroll
    for (int j = 0; j < kChunkCols; ++j) q[j / 4][j % 4] = __float_as_uint(f[j]);
  } else {
    q[0] = u32x4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
  }
  if (w.skip == 0 && D >= kChunkCols) {
#pragma unroll
    for (int k = 0; k < Chunk<DT>::kVecs; ++k) {
      if constexpr (ONCE) store_nt(p, k, q[k]);
      else reinterpret_cast<u32x4_row*>(p)[k] = q[k];
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < kChunkCols; ++j) {
    if (j < w.skip || j >= D) continue;
    if constexpr (DT == DT_F32) reinterpret_cast<uint32_t*>(p)[j] = q[j / 4][j % 4];
    else reinterpret_cast<uint16_t*>(p)[j] = (uint16_t)(q[0][j / 2] >> (16 * (j & 1)));
  }
}

// Lanes that share a row: a power of two, so that a workgroup holds a whole number of rows.
inline int lanes_per_row(int D) {
  const int chunks = (D + kChunkCols - 1) / kChunkCols;
  int lanes = kMinLanes;
  while (lanes < chunks && lanes < kEmbThreads) lanes *= 2;
  return lanes;
}

// A lane has eight columns; rows of few columns share a workgroup.  16384 x 4096 bf16: 33 us, 8.2 TB/s of rows read (the frequent
// ones from the last-level cache) and written; 9 rows: 2.9 us, a launch.
template <int DT, bool ONCE>
__global__ __launch_bounds__(kEmbThreads) void embedding_kernel(const void* table, const int32_t* ids, int n, int V,
                                                                int D, float scale, void* out, uint32_t* flags,
                                                                int lanes, long long first) {
  const long long i = (first + blockIdx.x) * (kEmbThreads / lanes) + threadIdx.x / lanes;
  if (i >= n) return;
  const int id = ids[i], l = threadIdx.x % lanes;
  const bool given = id >= 0 && id < V;
  const char* from = static_cast<const char*>(table) + (given ? (size_t)id * D * Elem<DT>::bytes : 0);
  char* to = static_cast<char*>(out) + (size_t)i * D * Elem<DT>::bytes;
  if (flags && l == 0) flags[i] = given || id == -1 ? 0 : SV_FLAG_BAD_TOKEN;
  for (int c = l; c * kChunkCols < D; c += lanes) {
    float f[kChunkCols] = {};
    if (given) {
      Chunk<DT> q;
      q.load(from, D, c);
      q.get(f);
    }
#pragma unroll
    for (int j = 0; j < kChunkCols; ++j) f[j] = given ? f[j] * scale : 0.f;
    store_chunk<DT, ONCE>(to, D, c, f);
  }
}

// ---------------------------------------------------------------------------
// stable sort of (token, position) by token, and the zeros of the table
// ---------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortPerLane = 4, kSortTile = kSortThreads * kSortPerLane;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kSortWaves = kSortThreads / kWave;

// A share of the table to be cleared by the workgroups of a launch from `first_block` on.
struct Clear {
  char* at;
  size_t bytes;                // 0: nothing (accumulating)
  int first_block;
};
constexpr size_t kClearBytes = 128 << 10;      // of one workgroup

__device__ __forceinline__ void clear_share(const Clear& z) {
  const size_t lo = (size_t)((int)blockIdx.x - z.first_block) * kClearBytes;
  const size_t n = lo < z.bytes ? min(kClearBytes, z.bytes - lo) : 0;
  const int vecs = (int)(n / 16);
  for (int i = threadIdx.x; i < vecs; i += blockDim.x) store_nt(z.at + lo, i, u32x4{0, 0, 0, 0});
  for (int i = vecs * 16 + threadIdx.x * 2; i < (int)n; i += blockDim.x * 2) *reinterpret_cast<uint16_t*>(z.at + lo + i) = 0;
}
inline unsigned clear_blocks(const Clear& z) { return (unsigned)((z.bytes + kClearBytes - 1) / kClearBytes); }

struct SortPass {
  const int32_t* ids;          // first pass: the tokens as given
  const uint32_t* key_in;      // later ones
  const int32_t* pos_in;
  uint32_t* key_out;
  int32_t* pos_out;
  int32_t* hist;               // [tiles, kDigits]
  int n, V, shift;
};

__device__ __forceinline__ uint32_t key_of_id(int id, int V) { return id >= 0 && id < V ? (uint32_t)id : (uint32_t)V; }
__device__ __forceinline__ uint32_t sort_key(const SortPass& p, int i) {
  return p.ids ? key_of_id(p.ids[i], p.V) : p.key_in[i];
}

// (65536 tokens: 7 us with a quarter of 131 MB of zeros beside it, 4.6 alone; the scatter 12 and 8.5.)
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const SortPass p, const Clear z) {
  if ((int)blockIdx.x >= z.first_block) return clear_share(z);
  __shared__ int count[kDigits];
  const int tid = threadIdx.x;
  if (tid < kDigits) count[tid] = 0;
  __syncthreads();
  const int base = blockIdx.x * kSortTile;
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    const int i = base + j * kSortThreads + tid;
    if (i < p.n) atomicAdd(&count[(sort_key(p, i) >> p.shift) & (kDigits - 1)], 1);
  }
  __syncthreads();
  if (tid < kDigits) p.hist[(size_t)blockIdx.x * kDigits + tid] = count[tid];
}

struct SortScratch {
  int count[kSortWaves][kDigits];
  int wave_sum[kSortWaves];
};

// Ranks of a tile's entries among those of their wavefront with the same digit; count[wave][digit] are the wavefront's numbers.
// Entries base .. base + 64 kSortPerLane - 1 of the tile are the wavefront's, `n` of the tile are there.
__device__ __forceinline__ void rank_digits(const uint32_t (&key)[kSortPerLane], int shift, int base, int n,
                                            int (&rank)[kSortPerLane], SortScratch& sm) {
  const int lane = threadIdx.x & 63;
  volatile int* mine = sm.count[threadIdx.x >> 6];
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    const bool on = base + j * kWave + lane < n;
    const int d = (key[j] >> shift) & (kDigits - 1);
    uint64_t same = __ballot(on);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
      const uint64_t set = __ballot((d >> b) & 1);
      same &= (d >> b) & 1 ? set : ~set;
    }
    const int below = __popcll(same & ((1ull << lane) - 1));
    const int so_far = mine[d];
    rank[j] = so_far + below;
    __builtin_amdgcn_wave_barrier();                   // (every lane has read before one of them writes)
    if (on && below == 0) mine[d] = so_far + __popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
}

// count[wave][digit] becomes where that wavefront's entries of the digit go: after those of smaller digits (`total` of each
// digit in all, of the lane whose number it is), of earlier tiles (`before`) and of earlier wavefronts.
__device__ __forceinline__ void place_digits(int before, int total, SortScratch& sm) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int scan = wave_scan_i32(tid < kDigits ? total : 0);
  if (lane == kWave - 1) sm.wave_sum[wave] = scan;
  __syncthreads();
  if (tid < kDigits) {
    int to = scan - total + before;
    for (int w = 0; w < wave; ++w) to += sm.wave_sum[w];
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = sm.count[w][tid];
      sm.count[w][tid] = to;
      to += c;
    }
  }
  __syncthreads();
}

__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(const SortPass p, int tiles, const Clear z) {
  if ((int)blockIdx.x >= z.first_block) return clear_share(z);
  __shared__ SortScratch sm;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < kSortWaves * kDigits; i += kSortThreads) (&sm.count[0][0])[i] = 0;
  __syncthreads();
  const int tile = blockIdx.x * kSortTile, base = wave * kSortPerLane * kWave, n = min(kSortTile, p.n - tile);
  uint32_t key[kSortPerLane];
  int pos[kSortPerLane], rank[kSortPerLane];
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    const int i = tile + base + j * kWave + lane;
    key[j] = i < p.n ? sort_key(p, i) : 0;
    pos[j] = i < p.n ? (p.ids ? i : p.pos_in[i]) : 0;
  }
  // entries of a digit in the tiles before this one, and in all: all loads under way before the first is used
  constexpr int kAhead = 16;
  int before = 0, total = 0;
  if (tid < kDigits) {
    for (int t0 = 0; t0 < tiles; t0 += kAhead) {
      int c[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) c[u] = t0 + u < tiles ? p.hist[(size_t)(t0 + u) * kDigits + tid] : 0;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        before += t0 + u < (int)blockIdx.x ? c[u] : 0;
        total += c[u];
      }
    }
  }
  rank_digits(key, p.shift, base, n, rank, sm);
  place_digits(before, total, sm);
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    if (base + j * kWave + lane >= n) continue;
    const int to = sm.count[wave][(key[j] >> p.shift) & (kDigits - 1)] + rank[j];
    p.key_out[to] = key[j];
    p.pos_out[to] = pos[j];
  }
}

// Up to a tile of tokens: all passes in one workgroup.
__global__ __launch_bounds__(kSortThreads) void sort_tile_kernel(const SortPass p, int bits, const Clear z) {
  if ((int)blockIdx.x >= z.first_block) return clear_share(z);
  __shared__ SortScratch sm;
  __shared__ uint32_t keys[kSortTile];
  __shared__ int32_t positions[kSortTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, base = wave * kSortPerLane * kWave;
  uint32_t key[kSortPerLane];
  int pos[kSortPerLane], rank[kSortPerLane];
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    pos[j] = base + j * kWave + lane;
    key[j] = pos[j] < p.n ? key_of_id(p.ids[pos[j]], p.V) : 0;
  }
#pragma unroll 1
  for (int shift = 0; shift < bits; shift += kDigitBits) {
    for (int i = tid; i < kSortWaves * kDigits; i += kSortThreads) (&sm.count[0][0])[i] = 0;
    __syncthreads();
    rank_digits(key, shift, base, p.n, rank, sm);
    __syncthreads();
    int total = 0;
    if (tid < kDigits)
      for (int w = 0; w < kSortWaves; ++w) total += sm.count[w][tid];
    place_digits(0, total, sm);
#pragma unroll
    for (int j = 0; j < kSortPerLane; ++j) {
      if (base + j * kWave + lane >= p.n) continue;
      const int to = sm.count[wave][(key[j] >> shift) & (kDigits - 1)] + rank[j];
      keys[to] = key[j];
      positions[to] = pos[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSortPerLane; ++j) {
      const int i = base + j * kWave + lane;
      if (i < p.n) { key[j] = keys[i]; pos[j] = positions[i]; }
    }
  }
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    const int i = base + j * kWave + lane;
    if (i < p.n) { p.key_out[i] = key[j]; p.pos_out[i] = pos[j]; }
  }
}

// ---------------------------------------------------------------------------
// sums
// ---------------------------------------------------------------------------
constexpr int kMaxGroups = kEmbThreads / kMinLanes;
constexpr int kMinPiece = 8, kMaxPiece = 64;
// Sorted positions that one group of lanes goes through, and the most a token may have to be summed by one group: 64, whose
// partial sums are a thirty-second of what is read, less where that would leave compute units without a workgroup
// (512 x 896 f32: 9.9 us with 16, 6.8 with 8).
inline int piece_of(int n, int D) {
  const long long groups = (long long)n * lanes_per_row(D) / kEmbThreads;        // positions by workgroups' groups
  int piece = kMinPiece;
  while (piece < kMaxPiece && groups >= 512LL * 2 * piece) piece *= 2;
  return piece;
}

struct GradRows {
  const void* g;
  void* table;
  const uint32_t* key;                  // sorted tokens
  const int32_t* pos;                   // their positions
  int32_t* begins;                      // [pieces] 2 * the token that begins in the piece and has more than a piece of positions,
                                        // + 1 if not with the piece's first; or -1
  int32_t* last;                        // [V] end of the sorted positions of such a token
  float* part;                          // [pieces, 2, D] sums over a piece of such a token: of the one that has the piece's
                                        // first position, and of another that begins in the piece
  int n, V, D, lanes, accumulate, piece;
  float scale;
};

template <int DTW, bool ONCE = true>
__device__ __forceinline__ void store_sum(const GradRows& a, uint32_t v, int c, float (&sum)[kChunkCols]) {
  char* to = static_cast<char*>(a.table) + (size_t)v * a.D * Elem<DTW>::bytes;
  float old[kChunkCols] = {};
  if (a.accumulate) {
    Chunk<DTW> q;
    q.load(to, a.D, c);
    q.get(old);
  }
#pragma unroll
  for (int j = 0; j < kChunkCols; ++j) sum[j] = __builtin_fmaf(sum[j], a.scale, old[j]);
  store_chunk<DTW, ONCE>(to, a.D, c, sum);
}

// What a group of lanes has to do: positions from .. to - 1 of the sorted list, the first token's sum (if it is joined) to slot
// 0 of the piece, the last one's (if it is) to slot 1.
struct Piece {
  int from, to;
  bool joins_first, joins_last;
};
// keys of the piece at key[0 ..], and a piece before and after it; ~0 where there is no position.
__device__ __forceinline__ Piece look_at(const uint32_t* key, int piece, uint32_t V) {
  auto end_of = [&](int lo, int hi, uint32_t k, bool after) {      // first entry of at least k, or above it
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (key[mid] < k || (after && key[mid] == k)) lo = mid + 1; else hi = mid;
    }
    return lo;
  };
  const int size = end_of(0, piece, V, false);         // of it, positions with a token
  Piece p = {0, size, false, false};
  if (size == 0) return p;
  const uint32_t k0 = key[0], k1 = key[size - 1];
  const int end0 = end_of(0, 2 * piece, k0, true);
  p.joins_first = end0 > piece || key[end0 - 1 - piece] == k0;
  if (key[-1] == k0 && !p.joins_first) p.from = min(end0, size);   // summed with the piece it begins in
  if (k1 == k0) {
    p.to = p.joins_first ? size : max(end0, p.from);
    if (key[-1] == k0 && !p.joins_first) p.to = p.from;
    return p;
  }
  const int begin1 = end_of(0, size, k1, false);
  p.joins_last = key[begin1 + piece] == k1;
  if (!p.joins_last) p.to = end_of(begin1, begin1 + piece, k1, true);
  return p;
}

// Goes through the sorted positions, the rows of eight of them under way at a time whatever tokens they belong to, and writes a
// token's row where its positions end.  65536 x 2048 bf16: 71 us, 4.5 TB/s of rows read in the order of their tokens and written.
template <int DTG, int DTW, bool ONCE>
__global__ __launch_bounds__(kEmbThreads) void embedding_grad_pieces_kernel(const GradRows a) {
  constexpr int kAhead = 8;
  __shared__ uint32_t key[(kMaxGroups + 2) * kMaxPiece + 1];
  __shared__ int32_t pos[(kMaxGroups + 1) * kMaxPiece];
  const int groups = kEmbThreads / a.lanes, piece = a.piece;
  const long long base = (long long)blockIdx.x * groups * piece;
  for (int j = threadIdx.x; j < (groups + 2) * piece; j += kEmbThreads) {
    const long long i = base - piece + j;
    key[j] = i >= 0 && i < a.n ? a.key[i] : ~0u;
    if (j >= piece) pos[j - piece] = i < a.n ? a.pos[i] : 0;
  }
  __syncthreads();
  const int l = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes;
  const uint32_t* k = key + (group + 1) * piece;
  const int32_t* at = pos + group * piece;
  const Piece p = look_at(k, piece, (uint32_t)a.V);
  if (l == 0 && base + group * piece < a.n)
    a.begins[base / piece + group] = p.joins_last ? (int)k[p.to - 1] * 2 + 1 : p.joins_first && k[-1] != k[0] ? (int)k[0] * 2 : -1;
  if (p.from >= p.to) return;
  const char* g = static_cast<const char*>(a.g);
  const size_t bytes = (size_t)a.D * Elem<DTG>::bytes;
  for (int c = l; c * kChunkCols < a.D; c += a.lanes) {
    float sum[kChunkCols] = {};
    for (int i = p.from; i < p.to; i += kAhead) {
      Chunk<DTG> q[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) q[u].template load<ONCE>(g + at[min(i + u, p.to - 1)] * bytes, a.D, c);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (i + u >= p.to) break;
        q[u].add_to(sum);
        const uint32_t v = k[i + u];
        if (i + u + 1 < p.to && k[i + u + 1] == v) continue;
        const bool first = p.joins_first && v == k[0], last = p.joins_last && i + u + 1 == p.to;
        if (first || last) {
          store_chunk<DT_F32>(a.part + ((size_t)(base / piece + group) * 2 + (first ? 0 : 1)) * a.D, a.D, c, sum);
          // its last position: what the join looks for
          if (l == 0 && c == 0 && k[i + u + 1] != v) a.last[v] = (int)(base + group * piece) + i + u + 1;
        } else {
          store_sum<DTW>(a, v, c, sum);
        }
#pragma unroll
        for (int j = 0; j < kChunkCols; ++j) sum[j] = 0.f;
      }
    }
  }
}

// Rows of tokens with more than a piece of positions.  A workgroup has kJoinPieces pieces and up to 64 chunks of their rows (a
// frequent token's partial sums are a megabyte, more than one compute unit reads in the time that the rest takes);
// its groups of lanes sum a run of a token's partial sums each, and those sums are added in order.
constexpr int kJoinThreads = 1024, kJoinPieces = 4, kJoinLanes = 64;
template <int DTW>
__global__ __launch_bounds__(kJoinThreads) void embedding_grad_join_kernel(const GradRows a) {
  __shared__ float sums[kJoinThreads][kChunkCols + 1];
  const int lanes = min(a.lanes, kJoinLanes), per_share = kJoinPieces * lanes, shares = kJoinThreads / per_share;
  const int share = threadIdx.x / per_share, t = threadIdx.x % per_share, c = blockIdx.y * lanes + t % lanes;
  const long long p0 = (long long)blockIdx.x * kJoinPieces + t / lanes;
  const int begins = p0 * a.piece < a.n && c * kChunkCols < a.D ? a.begins[p0] : -1;
  if (!__syncthreads_or(begins >= 0)) return;
  float sum[kChunkCols] = {};
  const uint32_t v = (uint32_t)begins >> 1;
  if (begins >= 0) {
    const int parts = (int)((a.last[v] - 1) / a.piece - p0) + 1, per = (parts + shares - 1) / shares;
    const int from = min(share * per, parts), to = min(from + per, parts);
    constexpr int kAhead = 8;
    for (int i = from; i < to; i += kAhead) {
      Chunk<DT_F32> q[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int j = min(i + u, to - 1);
        q[u].load(a.part + ((size_t)(p0 + j) * 2 + (j == 0 ? begins & 1 : 0)) * a.D, a.D, c);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (i + u < to) q[u].add_to(sum);
    }
  }
#pragma unroll
  for (int j = 0; j < kChunkCols; ++j) sums[threadIdx.x][j] = sum[j];
  __syncthreads();
  if (share > 0 || begins < 0) return;
  for (int s = 1; s < shares; ++s)
#pragma unroll
    for (int j = 0; j < kChunkCols; ++j) sum[j] += sums[s * per_share + t][j];
  store_sum<DTW>(a, v, c, sum);
}

// Few tokens: one launch.  Every workgroup looks through all tokens for those of its rows, orders them by row and position, and
// writes its rows, sums and zeros alike.  Rows of a group of lanes lie a grid apart, so that frequent tokens, whose numbers often
// lie together, are spread.  One group sums all of a token's rows, 0.13 us a row: with the limit at 256, that many of one token
// took 40 us here and 19 us sorted.  128 tokens, here and sorted: 7.5 and 20 us (5000 x 64 bf16), 14 and 20 us (32001 x 896 bf16),
// 100 and 120 us (152064 x 2048 bf16, 6.2 TB/s), 90 and 103 us (128256 x 1024 f32); all of one token 23 and 18 us (5000 x 64).
// A small table has one row a group (5000 x 64: 8.6 us in 20 workgroups of eight rounds, 7.5 in 157).
// Stores past the cache cost a float table 114 us where these take 50 (32000 x 2048): a lane's two vectors are half lines.
constexpr int kDirectTokens = 128, kRounds = 8, kDirectGroups = 1024;
static_assert(kDirectTokens <= kEmbThreads, "a lane has one token");

// Row v of the table: the sum of rows at[lo .. hi - 1] of the gradient, columns of lane l of `lanes`.
template <int DTG, int DTW>
__device__ __forceinline__ void write_row(const GradRows& a, uint32_t v, const uint16_t* at, int lo, int hi, int l, int lanes) {
  constexpr int kAhead = 16 / Chunk<DTG>::kVecs;
  const char* g = static_cast<const char*>(a.g);
  const size_t bytes = (size_t)a.D * Elem<DTG>::bytes;
  for (int c = l; c * kChunkCols < a.D; c += lanes) {
    float sum[kChunkCols] = {};
    for (int i = lo; i < hi; i += kAhead) {
      Chunk<DTG> q[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (i + u < hi) q[u].load(g + at[i + u] * bytes, a.D, c);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (i + u < hi) q[u].add_to(sum);
    }
    store_sum<DTW, false>(a, v, c, sum);
  }
}

// The positions of this workgroup's lanes that hit, in their order, to found[]; -> how many.  A wavefront's lanes call it together.
__device__ __forceinline__ int collect(bool here, int* count, uint16_t* found, int& to) {
  constexpr int kWaves = kEmbThreads / kWave;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t hit = __ballot(here);
  if (lane == 0) count[wave] = __popcll(hit);
  __syncthreads();
  int total = 0;
  to = __popcll(hit & ((1ull << lane) - 1));
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    to += w < wave ? count[w] : 0;
    total += count[w];
  }
  if (here) found[to] = (uint16_t)threadIdx.x;
  return total;
}

template <int DTG, int DTW>
__global__ __launch_bounds__(kEmbThreads) void embedding_grad_direct_kernel(const GradRows a, const int32_t* ids) {
  __shared__ uint16_t found[kDirectTokens], at[kDirectTokens], row_found[kDirectTokens];
  __shared__ uint16_t start[kRounds * kMaxGroups], end[kRounds * kMaxGroups];
  __shared__ int count[kEmbThreads / kWave];
  const int tid = threadIdx.x, groups = kEmbThreads / a.lanes;
  for (int r = tid; r < kRounds * groups; r += kEmbThreads) start[r] = end[r] = 0;
  const int id = tid < a.n ? ids[tid] : -1;
  const uint32_t unit = (uint32_t)max(id, 0) / (uint32_t)groups, round = unit / gridDim.x;
  const bool here = id >= 0 && id < a.V && unit - round * gridDim.x == blockIdx.x;
  int to;
  const int total = collect(here, count, found, to);
  if (here) row_found[to] = (uint16_t)(round * groups + (uint32_t)id % (uint32_t)groups);
  __syncthreads();
  if (tid < total) {
    const int r = row_found[tid];
    int smaller = 0, same = 0, earlier = 0;
    for (int m = 0; m < total; ++m) {
      const int o = row_found[m];
      smaller += o < r;
      same += o == r;
      earlier += o == r && m < tid;
    }
    at[smaller + earlier] = found[tid];
    if (earlier == 0) { start[r] = (uint16_t)smaller; end[r] = (uint16_t)(smaller + same); }
  }
  __syncthreads();
  const int l = tid % a.lanes, group = tid / a.lanes;
#pragma unroll 1
  for (int k = 0; k < kRounds; ++k) {
    const long long v = ((long long)k * gridDim.x + blockIdx.x) * groups + group;
    if (v >= a.V) return;
    write_row<DTG, DTW>(a, (uint32_t)v, at, start[k * groups + group], end[k * groups + group], l, a.lanes);
  }
}

// Few tokens added to a table: only their rows are touched, so there is a workgroup for each token, and the first of equal ones
// sums them all.  16 tokens of 152064 x 2048 bf16: 6.7 us (the host's call), 49 us by the table's rows as above, 18 us sorted.
template <int DTG, int DTW>
__global__ __launch_bounds__(kEmbThreads) void embedding_grad_add_kernel(const GradRows a, const int32_t* ids) {
  __shared__ uint16_t found[kDirectTokens];
  __shared__ int count[kEmbThreads / kWave];
  const int id = ids[blockIdx.x];
  if (id < 0 || id >= a.V) return;
  int to;
  const int total = collect((int)threadIdx.x < a.n && ids[min((int)threadIdx.x, a.n - 1)] == id, count, found, to);
  __syncthreads();
  if (found[0] == blockIdx.x) write_row<DTG, DTW>(a, (uint32_t)id, found, 0, total, threadIdx.x, kEmbThreads);
}

struct EmbeddingWs {
  uint32_t* key[2];
  int32_t* pos[2];
  int32_t* hist;
  int32_t *begins, *last;
  float* part;
  size_t bytes;
};
inline int sort_tiles(int n) { return (n + kSortTile - 1) / kSortTile; }
inline EmbeddingWs carve_embedding_ws(void* base, int n, int V, int D) {
  EmbeddingWs w = {};
  if (n <= kDirectTokens) return w;
  char* p = static_cast<char*>(base);
  size_t off = 0;
  const int piece = piece_of(n, D), pieces = (n + piece - 1) / piece;
  auto take = [&](size_t bytes) { char* q = p ? p + off : nullptr; off += ws_round(bytes); return q; };
  for (int i = 0; i < 2; ++i) {
    w.key[i] = reinterpret_cast<uint32_t*>(take((size_t)n * 4));
    w.pos[i] = reinterpret_cast<int32_t*>(take((size_t)n * 4));
  }
  w.hist = reinterpret_cast<int32_t*>(take((size_t)sort_tiles(n) * kDigits * 4));
  w.begins = reinterpret_cast<int32_t*>(take((size_t)pieces * 4));
  w.last = reinterpret_cast<int32_t*>(take((size_t)V * 4));
  w.part = reinterpret_cast<float*>(take((size_t)pieces * 2 * D * 4));
  w.bytes = off;
  return w;
}

template <int DTG, int DTW>
void launch_sums(const GradRows& a, const int32_t* ids, hipStream_t st) {
  if (a.n <= kDirectTokens && a.accumulate) {
    hipLaunchKernelGGL((embedding_grad_add_kernel<DTG, DTW>), dim3((unsigned)a.n), dim3(kEmbThreads), 0, st, a, ids);
    return;
  }
  if (a.n <= kDirectTokens) {
    const int units = (a.V + kEmbThreads / a.lanes - 1) / (kEmbThreads / a.lanes);
    const dim3 grid((unsigned)std::max((units + kRounds - 1) / kRounds, std::min(units, kDirectGroups)));
    hipLaunchKernelGGL((embedding_grad_direct_kernel<DTG, DTW>), grid, dim3(kEmbThreads), 0, st, a, ids);
    return;
  }
  const int per = kEmbThreads / a.lanes * a.piece;
  const dim3 grid((unsigned)(((long long)a.n + per - 1) / per));
  if ((long long)a.n * a.D * Elem<DTG>::bytes > kCacheBytes)           // 65536 x 2048 bf16: 71 us past the cache, 75 us through it
    hipLaunchKernelGGL((embedding_grad_pieces_kernel<DTG, DTW, true>), grid, dim3(kEmbThreads), 0, st, a);
  else
    hipLaunchKernelGGL((embedding_grad_pieces_kernel<DTG, DTW, false>), grid, dim3(kEmbThreads), 0, st, a);
  const int lanes = a.lanes < kJoinLanes ? a.lanes : kJoinLanes, chunks = (a.D + kChunkCols - 1) / kChunkCols;
  const int join_per = kJoinPieces * a.piece;
  const dim3 join((unsigned)(((long long)a.n + join_per - 1) / join_per), (unsigned)((chunks + lanes - 1) / lanes));
  hipLaunchKernelGGL(embedding_grad_join_kernel<DTW>, join, dim3(kJoinThreads), 0, st, a);
}

}  // namespace sv

extern "C" int sv_embedding(const void* table, const int32_t* ids, int n, int V, int D, int dtype, float scale,
                            void* out, uint32_t* flags_or_null, sv_stream_t stream) {
  using namespace sv;
  SV_REQUIRE(dtype == SV_F32 || dtype == SV_BF16, SV_ERR_DTYPE);
  SV_REQUIRE(n >= 0 && V >= 1 && D >= 1, SV_ERR_INVALID_ARG);
  SV_REQUIRE(V <= (1 << 24) && D <= (1 << 20), SV_ERR_TOO_LARGE);
  if (n == 0) return SV_OK;
  SV_REQUIRE(table && ids && out, SV_ERR_NULL);
  SV_REQUIRE(is_aligned(table, elem_bytes(dtype)) && is_aligned(out, elem_bytes(dtype)) && is_aligned(ids, 4) &&
                 is_aligned(flags_or_null, 4),
             SV_ERR_ALIGN);
  const int lanes = lanes_per_row(D), rows = kEmbThreads / lanes;
  hipStream_t st = as_stream(stream);
  const bool once = 2LL * n * D * elem_bytes(dtype) > kCacheBytes;      // 16384 x 4096 bf16: 33 us so, 42 us through the cache
  auto go = [&](auto kernel) {
    in_launches(((long long)n + rows - 1) / rows, kEmbThreads, [&](long long first, dim3 grid) {
      hipLaunchKernelGGL(kernel, grid, dim3(kEmbThreads), 0, st, table, ids, n, V, D, scale, out, flags_or_null, lanes, first);
    });
  };
  if (dtype == SV_F32) once ? go(embedding_kernel<DT_F32, true>) : go(embedding_kernel<DT_F32, false>);
  else once ? go(embedding_kernel<DT_BF16, true>) : go(embedding_kernel<DT_BF16, false>);
  return launch_status();
}

extern "C" size_t sv_embedding_grad_workspace_bytes(int n, int V, int D) {
  if (n < 0 || n > SV_EMBEDDING_MAX_TOKENS || V < 1 || V > (1 << 24) || D < 1 || D > (1 << 20)) return 0;
  const size_t need = sv::carve_embedding_ws(nullptr, n, V, D).bytes;
  return need < sv::kWsAlign ? sv::kWsAlign : need;
}

extern "C" int sv_embedding_grad(const void* grad_out, int dtype, const int32_t* ids, int n, int V, int D, float scale,
                                 void* grad_table, int table_dtype, int accumulate, void* ws, size_t ws_bytes,
                                 sv_stream_t stream) {
  using namespace sv;
  SV_REQUIRE((dtype == SV_F32 || dtype == SV_BF16) && (table_dtype == SV_F32 || table_dtype == SV_BF16), SV_ERR_DTYPE);
  SV_REQUIRE(n >= 0 && V >= 1 && D >= 1, SV_ERR_INVALID_ARG);
  SV_REQUIRE(n <= SV_EMBEDDING_MAX_TOKENS && V <= (1 << 24) && D <= (1 << 20), SV_ERR_TOO_LARGE);
  if (n == 0 && accumulate) return SV_OK;
  SV_REQUIRE(grad_table && (n == 0 || (grad_out && ids)), SV_ERR_NULL);
  SV_REQUIRE(is_aligned(grad_out, elem_bytes(dtype)) && is_aligned(grad_table, elem_bytes(table_dtype)) &&
                 is_aligned(ids, 4),
             SV_ERR_ALIGN);
  SV_REQUIRE(ws && is_aligned(ws, kWsAlign) && ws_bytes >= sv_embedding_grad_workspace_bytes(n, V, D), SV_ERR_WORKSPACE);
  hipStream_t st = as_stream(stream);
  const EmbeddingWs w = carve_embedding_ws(ws, n, V, D);
  int at = 0;
  if (n > kDirectTokens) {
    int bits = 1;
    while ((V >> bits) != 0) ++bits;                     // keys 0 .. V
    // the table's zeros, in equal shares to the launches of the sort
    const int passes = (bits + kDigitBits - 1) / kDigitBits, tiles = sort_tiles(n), launches = tiles == 1 ? 1 : 2 * passes;
    char* zeros = static_cast<char*>(grad_table);
    size_t left = accumulate ? 0 : (size_t)V * D * elem_bytes(table_dtype);
    const size_t least = launches * kClearBytes, share = (left + least - 1) / least * kClearBytes;      // (launches * share >= left)
    auto clear = [&](int first_block) {
      const Clear z = {zeros, share < left ? share : left, first_block};
      zeros += z.bytes;
      left -= z.bytes;
      return z;
    };
    const dim3 block(kSortThreads);
    if (tiles == 1) {
      const SortPass p = {ids, nullptr, nullptr, w.key[0], w.pos[0], nullptr, n, V, 0};
      const Clear z = clear(1);
      hipLaunchKernelGGL(sort_tile_kernel, dim3(1 + clear_blocks(z)), block, 0, st, p, bits, z);
    } else {
      for (int shift = 0; shift < bits; shift += kDigitBits) {
        const SortPass p = {shift == 0 ? ids : nullptr, w.key[at], w.pos[at], w.key[1 - at], w.pos[1 - at], w.hist, n, V, shift};
        const Clear z0 = clear(tiles);
        hipLaunchKernelGGL(sort_count_kernel, dim3(tiles + clear_blocks(z0)), block, 0, st, p, z0);
        const Clear z1 = clear(tiles);
        hipLaunchKernelGGL(sort_scatter_kernel, dim3(tiles + clear_blocks(z1)), block, 0, st, p, tiles, z1);
        at = 1 - at;
      }
    }
  }
  const GradRows a = {grad_out, grad_table, w.key[at], w.pos[at], w.begins, w.last, w.part, n, V, D, lanes_per_row(D),
                      accumulate != 0, piece_of(n, D), scale};
  if (dtype == SV_F32) {
    if (table_dtype == SV_F32) launch_sums<DT_F32, DT_F32>(a, ids, st);
    else launch_sums<DT_F32, DT_BF16>(a, ids, st);
  } else {
    if (table_dtype == SV_F32) launch_sums<DT_BF16, DT_F32>(a, ids, st);
    else launch_sums<DT_BF16, DT_BF16>(a, ids, st);
  }
  return launch_status();
}
