// sv_embedding: scaled rows of a table.  sv_embedding_grad: the gradient of that table.
//
// The gradient sorts the tokens (least significant digit first, kDigitBits bits a pass, stable) and then
// sums, for every row of the table, the rows of the token's positions in their order: no atomics
// on the result, the same bits from every call.  Positions whose id is no row sort behind all others.
#include "sv_device.hpp"
#include "sv_host.hpp"

namespace sv {

constexpr int kChunkCols = 8;           // columns of one lane: 16 bytes of bfloat16, 32 of float32
constexpr int kEmbThreads = 256;
constexpr int kMinLanes = 8;            // lanes of a row at least

// Columns 8c .. 8c + 7 of a row of D; columns past D are 0 and are not written.
template <int DT>
__device__ __forceinline__ void load_chunk(const void* row, int D, int c, float (&f)[kChunkCols]) {
  if ((c + 1) * kChunkCols <= D) {
    if constexpr (DT == DT_F32) {
      const u32x4 a = load_vec(row, 2 * c), b = load_vec(row, 2 * c + 1);
#pragma unroll
      for (int j = 0; j < 4; ++j) { f[j] = __uint_as_float(a[j]); f[4 + j] = __uint_as_float(b[j]); }
    } else {
      unpack<DT_BF16>(load_vec(row, c), f);
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < kChunkCols; ++j) f[j] = c * kChunkCols + j < D ? load_elem<DT>(row, c * kChunkCols + j) : 0.f;
}
template <int DT>
__device__ __forceinline__ void store_chunk(void* row, int D, int c, const float (&f)[kChunkCols]) {
  if constexpr (DT == DT_F32) {
    if ((c + 1) * kChunkCols <= D) {
      u32x4_row* p = reinterpret_cast<u32x4_row*>(row) + 2 * c;
      p[0] = u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
      p[1] = u32x4{__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])};
      return;
    }
#pragma unroll
    for (int j = 0; j < kChunkCols; ++j)
      if (c * kChunkCols + j < D) reinterpret_cast<float*>(row)[c * kChunkCols + j] = f[j];
  } else {
    const u32x4 q = {pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
    if ((c + 1) * kChunkCols <= D) {
      reinterpret_cast<u32x4_row*>(row)[c] = q;
      return;
    }
#pragma unroll
    for (int j = 0; j < kChunkCols; ++j)
      if (c * kChunkCols + j < D)
        reinterpret_cast<uint16_t*>(row)[c * kChunkCols + j] = (uint16_t)(q[j >> 1] >> (16 * (j & 1)));
  }
}

// Lanes that share a row: a power of two, so that a workgroup holds a whole number of rows.
inline int lanes_per_row(int D) {
  const int chunks = (D + kChunkCols - 1) / kChunkCols;
  int lanes = kMinLanes;
  while (lanes < chunks && lanes < kEmbThreads) lanes *= 2;
  return lanes;
}

template <int DT>
__global__ __launch_bounds__(kEmbThreads) void embedding_kernel(const void* table, const int32_t* ids, int n, int V,
                                                                int D, float scale, void* out, uint32_t* flags,
                                                                int lanes) {
  const long long i = (long long)blockIdx.x * (kEmbThreads / lanes) + threadIdx.x / lanes;
  if (i >= n) return;
  const int id = ids[i], l = threadIdx.x % lanes;
  const bool given = id >= 0 && id < V;
  const char* from = static_cast<const char*>(table) + (given ? (size_t)id * D * Elem<DT>::bytes : 0);
  char* to = static_cast<char*>(out) + (size_t)i * D * Elem<DT>::bytes;
  if (flags && l == 0) flags[i] = given || id == -1 ? 0 : SV_FLAG_BAD_TOKEN;
  for (int c = l; c * kChunkCols < D; c += lanes) {
    float f[kChunkCols] = {};
    if (given) load_chunk<DT>(from, D, c, f);
#pragma unroll
    for (int j = 0; j < kChunkCols; ++j) f[j] = given ? f[j] * scale : 0.f;
    store_chunk<DT>(to, D, c, f);
  }
}

// ---------------------------------------------------------------------------
// stable sort of (token, position) by token
// ---------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortPerLane = 4, kSortTile = kSortThreads * kSortPerLane;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kSortWaves = kSortThreads / kWave;

struct SortPass {
  const int32_t* ids;          // first pass: the tokens as given
  const uint32_t* key_in;      // later ones
  const int32_t* pos_in;
  uint32_t* key_out;
  int32_t* pos_out;
  int32_t* hist;               // [tiles, kDigits]
  int n, V, shift;
};

__device__ __forceinline__ uint32_t sort_key(const SortPass& p, int i) {
  if (!p.ids) return p.key_in[i];
  const int id = p.ids[i];
  return id >= 0 && id < p.V ? (uint32_t)id : (uint32_t)p.V;
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const SortPass p) {
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

// A wavefront owns kSortPerLane * 64 consecutive entries of the tile.
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(const SortPass p, int tiles) {
  __shared__ int count[kSortWaves][kDigits];
  __shared__ int wave_sum[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int i = tid; i < kSortWaves * kDigits; i += kSortThreads) (&count[0][0])[i] = 0;
  __syncthreads();
  const int base = blockIdx.x * kSortTile + wave * kSortPerLane * kWave;
  uint32_t key[kSortPerLane];
  int pos[kSortPerLane], rank[kSortPerLane];
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    const int i = base + j * kWave + lane;
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
  volatile int* mine = count[wave];
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    const bool on = base + j * kWave + lane < p.n;
    const int d = (key[j] >> p.shift) & (kDigits - 1);
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
  __syncthreads();
  // where a digit's entries of this tile start, and each wavefront's within them
  int own = 0;
  const int scan = wave_scan_i32(total);
  if (lane == kWave - 1) wave_sum[wave] = scan;
  __syncthreads();
  int start = scan - total;
  for (int w = 0; w < wave; ++w) start += wave_sum[w];
  if (tid < kDigits) {
    own = start + before;
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = count[w][tid];
      count[w][tid] = own;
      own += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    if (base + j * kWave + lane >= p.n) continue;
    const int to = count[wave][(key[j] >> p.shift) & (kDigits - 1)] + rank[j];
    p.key_out[to] = key[j];
    p.pos_out[to] = pos[j];
  }
}

// ---------------------------------------------------------------------------
// sums
// ---------------------------------------------------------------------------
constexpr int kRounds = 8;              // rows of the table of one group of lanes
constexpr int kMaxGroups = kEmbThreads / kMinLanes, kMaxRows = kRounds * kMaxGroups;
constexpr int kPiece = 64;              // sorted positions summed by one group of lanes; a token with more is joined from pieces
constexpr int kDirectTokens = 1024;     // up to here every workgroup looks through all tokens itself

// Row of the table that group `group` of workgroup `block` has in round k: frequent tokens, whose numbers
// often lie together, are spread over the workgroups.
__device__ __forceinline__ long long row_of(int block, int group, int groups, int k) {
  return ((long long)k * gridDim.x + block) * groups + group;
}

struct GradRows {
  const void* g;
  void* table;
  const int32_t* ids;                   // direct form: the tokens as given
  const uint32_t* key;                  // sorted tokens
  const int32_t* pos;                   // their positions
  int32_t *first, *last;                // [V] range of a token's sorted positions; of tokens that occur
  float* part;                          // [pieces, 2, D] sums of a piece over a token that began before it / goes on after it
  int n, V, D, lanes, accumulate;
  float scale;
};

// sum += the rows of positions at(lo) .. at(hi - 1), in this order; eight 16-byte loads of a lane are under way at a time.
template <int DT, class At>
__device__ __forceinline__ void add_rows(const GradRows& a, int c, int lo, int hi, At&& at, float (&sum)[kChunkCols]) {
  constexpr int kVecs = kChunkCols / Elem<DT>::per_vec, kAhead = 8 / kVecs;
  const char* g = static_cast<const char*>(a.g);
  const size_t bytes = (size_t)a.D * Elem<DT>::bytes;
  if ((c + 1) * kChunkCols > a.D) {                    // the last columns of a row that is no multiple of 8
    for (int i = lo; i < hi; ++i) {
      float f[kChunkCols];
      load_chunk<DT>(g + at(i) * bytes, a.D, c, f);
#pragma unroll
      for (int j = 0; j < kChunkCols; ++j) sum[j] += f[j];
    }
    return;
  }
  auto add = [&](const u32x4 (&q)[kVecs]) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) {
      float f[Elem<DT>::per_vec];
      unpack<DT>(q[k], f);
#pragma unroll
      for (int j = 0; j < Elem<DT>::per_vec; ++j) sum[k * Elem<DT>::per_vec + j] += f[j];
    }
  };
  auto load = [&](int i, u32x4 (&q)[kVecs]) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) q[k] = load_vec(g + at(i) * bytes, c * kVecs + k);
  };
  int i = lo;
  for (; i + kAhead <= hi; i += kAhead) {
    u32x4 q[kAhead][kVecs];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) load(i + u, q[u]);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) add(q[u]);
  }
  if (i < hi) {                                        // the last, partial round
    u32x4 q[kAhead - 1][kVecs];
#pragma unroll
    for (int u = 0; u < kAhead - 1; ++u)
      if (i + u < hi) load(i + u, q[u]);
#pragma unroll
    for (int u = 0; u < kAhead - 1; ++u)
      if (i + u < hi) add(q[u]);
  }
}

template <int DTW>
__device__ __forceinline__ void store_sum(const GradRows& a, int v, int c, float (&sum)[kChunkCols]) {
  char* to = static_cast<char*>(a.table) + (size_t)v * a.D * Elem<DTW>::bytes;
  float old[kChunkCols] = {};
  if (a.accumulate) load_chunk<DTW>(to, a.D, c, old);
#pragma unroll
  for (int j = 0; j < kChunkCols; ++j) sum[j] = __builtin_fmaf(sum[j], a.scale, old[j]);
  store_chunk<DTW>(to, a.D, c, sum);
}

// Few tokens: one launch.  A workgroup picks the tokens of its rows out of all, in the order of their positions.
template <int DTG, int DTW>
__global__ __launch_bounds__(kEmbThreads) void embedding_grad_direct_kernel(const GradRows a) {
  constexpr int kWaves = kEmbThreads / kWave, kLooks = kDirectTokens / kEmbThreads;
  __shared__ uint32_t found[kDirectTokens];            // row of the workgroup << 16 | position
  __shared__ uint16_t pos[kDirectTokens];              // positions by row, then by position
  __shared__ uint16_t start[kMaxRows], end[kMaxRows];
  __shared__ int count[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int groups = kEmbThreads / a.lanes;
  for (int r = threadIdx.x; r < kRounds * groups; r += kEmbThreads) start[r] = end[r] = 0;
  // a wavefront looks through a run of tokens
  uint64_t hit[kLooks];
  int row[kLooks], mine = 0;
#pragma unroll
  for (int j = 0; j < kLooks; ++j) {
    const int i = (wave * kLooks + j) * kWave + lane;
    const int id = i < a.n ? a.ids[i] : -1;
    const uint32_t unit = (uint32_t)max(id, 0) / (uint32_t)groups, k = unit / gridDim.x;
    row[j] = (int)k * groups + max(id, 0) % groups;
    hit[j] = __ballot(id >= 0 && id < a.V && unit - k * gridDim.x == blockIdx.x);
    mine += __popcll(hit[j]);
  }
  if (lane == 0) count[wave] = mine;
  __syncthreads();
  int to = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    to += w < wave ? count[w] : 0;
    total += count[w];
  }
#pragma unroll
  for (int j = 0; j < kLooks; ++j) {
    if (hit[j] >> lane & 1)
      found[to + __popcll(hit[j] & ((1ull << lane) - 1))] = (uint32_t)row[j] << 16 | ((wave * kLooks + j) * kWave + lane);
    to += __popcll(hit[j]);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < total; i += kEmbThreads) {
    const uint32_t f = found[i], r = f >> 16;
    int smaller = 0, same = 0, earlier = 0;
    for (int m = 0; m < total; ++m) {
      const uint32_t o = found[m] >> 16;
      smaller += o < r;
      same += o == r;
      earlier += o == r && m < i;
    }
    pos[smaller + earlier] = (uint16_t)f;
    if (earlier == 0) { start[r] = (uint16_t)smaller; end[r] = (uint16_t)(smaller + same); }
  }
  __syncthreads();
  const int l = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes;
  for (int k = 0; k < kRounds; ++k) {
    const long long v = row_of(blockIdx.x, group, groups, k);
    if (v >= a.V) break;
    const int lo = start[k * groups + group], hi = end[k * groups + group];
    if (lo == hi && a.accumulate) continue;
    for (int c = l; c * kChunkCols < a.D; c += a.lanes) {
      float sum[kChunkCols] = {};
      add_rows<DTG>(a, c, lo, hi, [&](int i) { return (size_t)pos[i]; }, sum);
      store_sum<DTW>(a, (int)v, c, sum);
    }
  }
}

// Many tokens, first launch: where the tokens' sorted positions begin and end, and the sums of pieces of those
// that have more than kPiece.  Such a token is in a piece from its first position on, or up to its last.
template <int DTG>
__global__ __launch_bounds__(kEmbThreads) void embedding_grad_pieces_kernel(const GradRows a) {
  __shared__ uint32_t key[kMaxGroups * kPiece];
  __shared__ int32_t pos[kMaxGroups * kPiece];
  const int pieces = kEmbThreads / a.lanes;            // of the workgroup
  const long long base = (long long)blockIdx.x * pieces * kPiece;
  for (int j = threadIdx.x; j < pieces * kPiece && base + j < a.n; j += kEmbThreads) {
    const int i = (int)(base + j);
    const uint32_t k = a.key[i];
    const uint32_t left = i > 0 ? a.key[i - 1] : ~0u, right = i < a.n - 1 ? a.key[i + 1] : ~0u;
    key[j] = k;
    pos[j] = a.pos[i];
    if (k >= (uint32_t)a.V) continue;
    if (left != k) a.first[k] = i;
    if (right != k) a.last[k] = i + 1;
  }
  __syncthreads();
  const int l = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes;
  const long long lo = base + group * kPiece;
  if (lo >= a.n) return;
  const int size = (int)min((long long)kPiece, a.n - lo);
  const uint32_t* mine = key + group * kPiece;
  auto sum_piece = [&](int from, int to, int slot) {
    for (int c = l; c * kChunkCols < a.D; c += a.lanes) {
      float sum[kChunkCols] = {};
      add_rows<DTG>(a, c, from, to, [&](int i) { return (size_t)pos[group * kPiece + i]; }, sum);
      store_chunk<DT_F32>(a.part + ((size_t)(lo / kPiece) * 2 + slot) * a.D, a.D, c, sum);
    }
  };
  auto search = [&](uint32_t k) {                      // first entry of the piece with a key of at least k
    int x = 0, y = size;
    while (x < y) {
      const int mid = (x + y) / 2;
      if (mine[mid] < k) x = mid + 1; else y = mid;
    }
    return x;
  };
  auto has = [&](long long i, uint32_t k) { return i >= 0 && i < a.n && a.key[i] == k; };
  const uint32_t k0 = mine[0], k1 = mine[size - 1];
  const int to = search(k0 + 1), from = search(k1);
  // more than kPiece positions: the first token's begin before the piece, or fill it and go on
  if (k0 < (uint32_t)a.V && (has(lo + to - 1 - kPiece, k0) || (to == kPiece && has(lo + kPiece, k0)))) sum_piece(0, to, 0);
  if (to < size && k1 < (uint32_t)a.V && has(lo + from + kPiece, k1)) sum_piece(from, size, 1);
}

// Second launch: every row of the table.
template <int DTG, int DTW>
__global__ __launch_bounds__(kEmbThreads) void embedding_grad_rows_kernel(const GradRows a) {
  __shared__ int start[kMaxRows], end[kMaxRows];
  const int groups = kEmbThreads / a.lanes;
  for (int r = threadIdx.x; r < kRounds * groups; r += kEmbThreads) {
    // what the arrays hold for a token that does not occur is from elsewhere: no sorted position has that token
    const long long v = row_of(blockIdx.x, r % groups, groups, r / groups);
    const int lo = v < a.V ? a.first[v] : -1;
    const bool occurs = lo >= 0 && lo < a.n && a.key[lo] == (uint32_t)v;
    start[r] = occurs ? lo : 0;
    end[r] = occurs ? a.last[v] : 0;
  }
  __syncthreads();
  const int l = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes;
  for (int k = 0; k < kRounds; ++k) {
    const long long v = row_of(blockIdx.x, group, groups, k);
    if (v >= a.V) break;
    const int lo = start[k * groups + group], hi = end[k * groups + group];
    if (lo == hi && a.accumulate) continue;
    for (int c = l; c * kChunkCols < a.D; c += a.lanes) {
      float sum[kChunkCols] = {};
      if (hi - lo <= kPiece) {
        add_rows<DTG>(a, c, lo, hi, [&](int i) { return (size_t)a.pos[i]; }, sum);
      } else {
        GradRows parts = {};
        parts.g = a.part;
        parts.D = a.D;
        const int p0 = lo / kPiece, slot0 = lo % kPiece != 0;
        add_rows<DT_F32>(parts, c, p0, (hi - 1) / kPiece + 1, [&](int p) { return (size_t)p * 2 + (p == p0 ? slot0 : 0); },
                         sum);
      }
      store_sum<DTW>(a, (int)v, c, sum);
    }
  }
}

struct EmbeddingWs {
  uint32_t* key[2];
  int32_t* pos[2];
  int32_t* hist;
  int32_t *first, *last;
  float* part;
  size_t bytes;
};
inline int sort_tiles(int n) { return (n + kSortTile - 1) / kSortTile; }
inline EmbeddingWs carve_embedding_ws(void* base, int n, int V, int D) {
  EmbeddingWs w = {};
  if (n <= kDirectTokens) return w;
  char* p = static_cast<char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) { char* q = p ? p + off : nullptr; off += ws_round(bytes); return q; };
  for (int i = 0; i < 2; ++i) {
    w.key[i] = reinterpret_cast<uint32_t*>(take((size_t)n * 4));
    w.pos[i] = reinterpret_cast<int32_t*>(take((size_t)n * 4));
  }
  w.hist = reinterpret_cast<int32_t*>(take((size_t)sort_tiles(n) * kDigits * 4));
  w.first = reinterpret_cast<int32_t*>(take((size_t)V * 4));
  w.last = reinterpret_cast<int32_t*>(take((size_t)V * 4));
  w.part = reinterpret_cast<float*>(take((size_t)((n + kPiece - 1) / kPiece) * 2 * D * 4));
  w.bytes = off;
  return w;
}

template <int DTG>
void launch_grad_rows(const GradRows& a, int table_dtype, hipStream_t st) {
  const int rows = kEmbThreads / a.lanes * kRounds;
  const dim3 grid((unsigned)((a.V + rows - 1) / rows)), block(kEmbThreads);
  if (!a.key) {                                          // (of no tokens at all the list may be NULL as well)
    if (table_dtype == SV_F32) hipLaunchKernelGGL((embedding_grad_direct_kernel<DTG, DT_F32>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((embedding_grad_direct_kernel<DTG, DT_BF16>), grid, block, 0, st, a);
    return;
  }
  const int per = kEmbThreads / a.lanes * kPiece;
  hipLaunchKernelGGL(embedding_grad_pieces_kernel<DTG>, dim3((unsigned)((a.n + per - 1) / per)), block, 0, st, a);
  if (table_dtype == SV_F32) hipLaunchKernelGGL((embedding_grad_rows_kernel<DTG, DT_F32>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((embedding_grad_rows_kernel<DTG, DT_BF16>), grid, block, 0, st, a);
}

}  // namespace sv

extern "C" int sv_embedding(const void* table, const int32_t* ids, int n, int V, int D, int dtype, float scale,
                            void* out, uint32_t* flags_or_null, sv_stream_t stream) {
  using namespace sv;
  SV_REQUIRE(dtype == SV_F32 || dtype == SV_BF16, SV_ERR_DTYPE);
  SV_REQUIRE(n >= 0 && V >= 1 && D >= 1, SV_ERR_INVALID_ARG);
  SV_REQUIRE(V <= (1 << 24) && D <= (1 << 24), SV_ERR_TOO_LARGE);
  if (n == 0) return SV_OK;
  SV_REQUIRE(table && ids && out, SV_ERR_NULL);
  SV_REQUIRE(is_aligned(table, elem_bytes(dtype)) && is_aligned(out, elem_bytes(dtype)) && is_aligned(ids, 4) &&
                 is_aligned(flags_or_null, 4),
             SV_ERR_ALIGN);
  const int lanes = lanes_per_row(D), rows = kEmbThreads / lanes;
  const dim3 grid((unsigned)(((long long)n + rows - 1) / rows)), block(kEmbThreads);
  hipStream_t st = as_stream(stream);
  if (dtype == SV_F32)
    hipLaunchKernelGGL(embedding_kernel<DT_F32>, grid, block, 0, st, table, ids, n, V, D, scale, out, flags_or_null, lanes);
  else
    hipLaunchKernelGGL(embedding_kernel<DT_BF16>, grid, block, 0, st, table, ids, n, V, D, scale, out, flags_or_null, lanes);
  return launch_status();
}

extern "C" size_t sv_embedding_grad_workspace_bytes(int n, int V, int D) {
  if (n < 0 || n > SV_EMBEDDING_MAX_TOKENS || V < 1 || V > (1 << 24) || D < 1 || D > (1 << 24)) return 0;
  const size_t need = sv::carve_embedding_ws(nullptr, n, V, D).bytes;
  return need < sv::kWsAlign ? sv::kWsAlign : need;
}

extern "C" int sv_embedding_grad(const void* grad_out, int dtype, const int32_t* ids, int n, int V, int D, float scale,
                                 void* grad_table, int table_dtype, int accumulate, void* ws, size_t ws_bytes,
                                 sv_stream_t stream) {
  using namespace sv;
  SV_REQUIRE((dtype == SV_F32 || dtype == SV_BF16) && (table_dtype == SV_F32 || table_dtype == SV_BF16), SV_ERR_DTYPE);
  SV_REQUIRE(n >= 0 && V >= 1 && D >= 1, SV_ERR_INVALID_ARG);
  SV_REQUIRE(n <= SV_EMBEDDING_MAX_TOKENS && V <= (1 << 24) && D <= (1 << 24), SV_ERR_TOO_LARGE);
  if (n == 0 && accumulate) return SV_OK;
  SV_REQUIRE(grad_table && (n == 0 || (grad_out && ids)), SV_ERR_NULL);
  SV_REQUIRE(is_aligned(grad_out, elem_bytes(dtype)) && is_aligned(grad_table, elem_bytes(table_dtype)) &&
                 is_aligned(ids, 4),
             SV_ERR_ALIGN);
  SV_REQUIRE(ws && is_aligned(ws, kWsAlign) && ws_bytes >= sv_embedding_grad_workspace_bytes(n, V, D), SV_ERR_WORKSPACE);
  hipStream_t st = as_stream(stream);
  GradRows a = {grad_out, grad_table, ids, nullptr, nullptr, nullptr, nullptr, nullptr, n, V, D, lanes_per_row(D),
                accumulate != 0, scale};
  if (n > kDirectTokens) {
    const EmbeddingWs w = carve_embedding_ws(ws, n, V, D);
    int bits = 1, at = 0;
    while ((V >> bits) != 0) ++bits;                     // keys 0 .. V
    for (int shift = 0; shift < bits; shift += kDigitBits) {
      const SortPass p = {shift == 0 ? ids : nullptr, w.key[at], w.pos[at], w.key[1 - at], w.pos[1 - at], w.hist, n, V, shift};
      const dim3 grid((unsigned)sort_tiles(n)), block(kSortThreads);
      hipLaunchKernelGGL(sort_count_kernel, grid, block, 0, st, p);
      hipLaunchKernelGGL(sort_scatter_kernel, grid, block, 0, st, p, sort_tiles(n));
      at = 1 - at;
    }
    a.key = w.key[at]; a.pos = w.pos[at]; a.first = w.first; a.last = w.last; a.part = w.part;
  }
  if (dtype == SV_F32) launch_grad_rows<DT_F32>(a, table_dtype, st);
  else launch_grad_rows<DT_BF16>(a, table_dtype, st);
  return launch_status();
}
