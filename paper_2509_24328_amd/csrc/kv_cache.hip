// sv_cache_write, sv_cache_read: keys and values of new tokens into the pages of a cache, and rows of a cache back.
// A cache in 8 bits holds e4m3 numbers and a float32 scale for every token and head, amax / 448 (not below 2^-126; 1 where all
// columns are 0): the largest column of a head is then as well resolved as e4m3 resolves anything, whatever the layer's range, and a
// row costs 4 bytes more.  A head that holds a NaN or an infinity has the scale NaN and reads back as NaN.
// A workgroup has one token, four from 4096 tokens on: its place and angles once, then a head for every eight lanes, so that queries, keys
// and values share one launch and one lookup.  What bounds it: one user's or one step's tokens, a chain of loads (offsets and lengths, the page,
// the head) and the store (64 x 9 tokens, 48 heads of 128 bf16 columns into 8 bits: 8.2 us); a prompt, the memory (4096 tokens, 24 heads of 80
// float32 columns: 16 us, 3.9 TB/s; 5096 tokens back: 12.5 us, 4.2 TB/s).
#include "paged.hpp"
#include "rope.hpp"

namespace sv {

struct CacheArgs {
  const char *q, *k, *v;
  char* q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;   // bytes from row to row
  int Hq, tokens;
  Rows rows;
  Pages pages;
  const double* freq;                                   // null: nothing is turned
  RopeShape sh, plain;                                  // of queries and keys; of values
  double amplitude;
  char *k_cache, *v_cache;
  float *k_scale, *v_scale;
  uint32_t* flags;
};

// The maximum over the lanes of a group of eight.
__device__ __forceinline__ float group_max(float v) {
  v = fmaxf(v, lane_xor<1>(v));
  v = fmaxf(v, lane_xor<2>(v));
  return fmaxf(v, lane_xor<4>(v));
}

__device__ __forceinline__ uint32_t pack_f8(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// A row of the cache: first its largest magnitude, then its codes.  The row is turned twice rather than kept: it is in the cache the
// second time, and keys and values are the smaller part of what a call writes.
template <int DT, bool PAIRS>
__device__ __forceinline__ void write_f8(const void* row, const RopeShape& sh, const CosSin* cs, int lane, char* to,
                                         float* scale_at) {
  constexpr int EPV = Elem<DT>::per_vec;
  float top = 0.f;
  bool bad = false;
  turn_head<DT, PAIRS>(row, sh, cs, lane, false, [&](int, int n, const float (&f)[EPV]) {
#pragma unroll
    for (int e = 0; e < EPV; ++e) {
      if (e >= n) continue;
      top = fmaxf(top, fabsf(f[e]));
      bad |= !(fabsf(f[e]) < INFINITY);
    }
  });
  top = group_max(bad ? INFINITY : top);
  const bool nan = top == INFINITY;
  const float scale = nan ? NAN : (top > 0.f ? fmaxf(top / 448.f, 1.17549435e-38f) : 1.f);
  turn_head<DT, PAIRS>(row, sh, cs, lane, false, [&](int at, int n, const float (&f)[EPV]) {
    float c[EPV];
#pragma unroll
    for (int e = 0; e < EPV; ++e) c[e] = nan ? 0.f : fminf(fmaxf(f[e] / scale, -448.f), 448.f);
    uint32_t w[EPV / 4];
#pragma unroll
    for (int e = 0; e < EPV; e += 4) w[e / 4] = pack_f8(c[e], c[e + 1], c[e + 2], c[e + 3]);
    if (n >= EPV) {
      typedef uint32_t words __attribute__((ext_vector_type(EPV / 4), aligned(1)));
      __builtin_memcpy(to + at, w, EPV);
    } else {
#pragma unroll
      for (int e = 0; e < EPV; ++e)
        if (e < n) to[at + e] = (char)(w[e / 4] >> (8 * (e % 4)));
    }
  });
  if (lane == 0) *scale_at = scale;
}

template <int DT, bool PAIRS, bool F8>
__global__ void __launch_bounds__(kRopeThreads) cache_write_kernel(CacheArgs a) {
  constexpr int EPV = Elem<DT>::per_vec;
  extern __shared__ CosSin cs[];                       // [tokens][pitch]
  __shared__ int sh_b[4], sh_pos[4];
  __shared__ int64_t sh_row[4];
  const int r0 = blockIdx.x * a.tokens, half = a.sh.half, D = a.sh.D;
  const int nt = min(a.tokens, a.rows.n_rows - r0);
  const double freq0 = half && (int)threadIdx.x < nt * half ? a.freq[threadIdx.x % half] : 0.0;   // (asked for ahead of the places)
  if (threadIdx.x < kWave)
    for (int t = 0; t < nt; ++t) {
      const Place p = place_of_row(a.rows, r0 + t);
      const int64_t at = p.b < 0 ? -1 : cache_row(a.pages, p.b, p.position);
      if (threadIdx.x == 0) {
        sh_b[t] = p.b;
        sh_pos[t] = p.position;
        sh_row[t] = at;
        if (p.b >= 0 && a.flags) a.flags[r0 + t] = at < 0 ? SV_FLAG_BAD_PAGE : 0;
      }
    }
  __syncthreads();
  if (half) {
    for (int k = threadIdx.x; k < nt * half; k += kRopeThreads) {
      const int t = k / half;
      if (sh_b[t] >= 0)
        cs[t * a.sh.pitch + angle_at<EPV>(k - t * half)] =
            cos_sin((double)sh_pos[t] * (k < kRopeThreads ? freq0 : a.freq[k - t * half]), a.amplitude);
    }
    __syncthreads();
  }
  const int lane = threadIdx.x % kRopeLanes, H = a.Hq + 2 * a.pages.heads;
  constexpr int e_in = Elem<DT>::bytes, e_out = F8 ? 1 : e_in;
  for (int k = threadIdx.x / kRopeLanes; k < nt * H; k += kRopeGroups) {
    const int t = k / H, h = k - t * H;
    if (sh_b[t] < 0) continue;
    const int64_t r = r0 + t;
    const CosSin* c = cs + t * a.sh.pitch;
    if (h < a.Hq) {
      const char* from = a.q + r * a.q_stride + (int64_t)h * D * e_in;
      char* to = a.q_out + r * a.q_out_stride + (int64_t)h * D * e_in;
      turn_head<DT, PAIRS>(from, a.sh, c, lane, a.q == a.q_out,
                           [&](int at, int n, const float (&f)[EPV]) { store_some<DT>(to, at, n, f); });
      continue;
    }
    if (sh_row[t] < 0) continue;
    const bool value = h >= a.Hq + a.pages.heads;
    const int hk = h - a.Hq - (value ? a.pages.heads : 0);
    const char* from = (value ? a.v + r * a.v_stride : a.k + r * a.k_stride) + (int64_t)hk * D * e_in;
    const int64_t at_row = sh_row[t] + (int64_t)hk * (int)a.pages.page.d;
    char* to = (value ? a.v_cache : a.k_cache) + at_row * D * e_out;
    const RopeShape sh = value ? a.plain : a.sh;
    if constexpr (F8) {
      write_f8<DT, PAIRS>(from, sh, c, lane, to, (value ? a.v_scale : a.k_scale) + at_row);
    } else {
      turn_head<DT, PAIRS>(from, sh, c, lane, false,
                           [&](int at, int n, const float (&f)[EPV]) { store_some<DT>(to, at, n, f); });
    }
  }
}

struct ReadArgs {
  char *k, *v;
  int64_t k_stride, v_stride;
  int tokens, D;
  Rows rows;
  Pages pages;
  const char *k_cache, *v_cache;
  const float *k_scale, *v_scale;
  uint32_t* flags;
};

template <int DT, bool F8>
__global__ void __launch_bounds__(kRopeThreads) cache_read_kernel(ReadArgs a) {
  constexpr int EPV = Elem<DT>::per_vec, e_out = Elem<DT>::bytes, e_in = F8 ? 1 : e_out;
  __shared__ int sh_b[4];
  __shared__ int64_t sh_row[4];
  const int r0 = blockIdx.x * a.tokens, D = a.D, heads = a.pages.heads;
  const int nt = min(a.tokens, a.rows.n_rows - r0);
  if (threadIdx.x < kWave)
    for (int t = 0; t < nt; ++t) {
      const Place p = place_of_row(a.rows, r0 + t);
      const int64_t at = p.b < 0 ? -1 : cache_row(a.pages, p.b, p.position);
      if (threadIdx.x == 0) {
        sh_b[t] = p.b;
        sh_row[t] = at;
        if (p.b >= 0 && a.flags) a.flags[r0 + t] = at < 0 ? SV_FLAG_BAD_PAGE : 0;
      }
    }
  __syncthreads();
  const int lane = threadIdx.x % kRopeLanes, H = 2 * heads;
  for (int k = threadIdx.x / kRopeLanes; k < nt * H; k += kRopeGroups) {
    const int t = k / H, h = k - t * H;
    if (sh_b[t] < 0) continue;
    const int64_t r = r0 + t;
    const bool value = h >= heads, bad = sh_row[t] < 0;
    const int hk = value ? h - heads : h;
    char* to = (value ? a.v + r * a.v_stride : a.k + r * a.k_stride) + (int64_t)hk * D * e_out;
    const int64_t at_row = bad ? 0 : sh_row[t] + (int64_t)hk * (int)a.pages.page.d;
    const char* from = (value ? a.v_cache : a.k_cache) + at_row * D * e_in;
    float scale = 1.f;
    if constexpr (F8) scale = bad ? 1.f : (value ? a.v_scale : a.k_scale)[at_row];
    for (int at = lane * EPV; at < D; at += kRopeLanes * EPV) {
      const int n = min(EPV, D - at);
      float f[EPV];
      if (bad) {
#pragma unroll
        for (int e = 0; e < EPV; ++e) f[e] = NAN;
      } else if constexpr (F8) {
        uint32_t w[EPV / 4] = {};
        if (n >= EPV) {
          __builtin_memcpy(w, from + at, EPV);
        } else {
#pragma unroll
          for (int e = 0; e < EPV; ++e)
            if (e < n) w[e / 4] |= (uint32_t)(uint8_t)from[at + e] << (8 * (e % 4));
        }
#pragma unroll
        for (int e = 0; e < EPV; e += 4) {
          const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[e / 4], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[e / 4], true);
          f[e] = lo[0] * scale;
          f[e + 1] = lo[1] * scale;
          f[e + 2] = hi[0] * scale;
          f[e + 3] = hi[1] * scale;
        }
      } else {
        load_some<DT>(from, at, n, f);
      }
      store_some<DT>(to, at, n, f);
    }
  }
}

// Rows of a workgroup: one where the rows are few (their latency counts), four where there are enough of them for several workgroups
// to a compute unit.
inline int tokens_of(int n_rows) { return n_rows >= 4096 ? 4 : 1; }

inline int check_cache(const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale, int cache_dtype,
                       int dtype) {
  SV_REQUIRE(k_cache && v_cache, SV_ERR_NULL);
  const int e = cache_dtype == SV_F8 ? 1 : elem_bytes(dtype);
  SV_REQUIRE(is_aligned(k_cache, e) && is_aligned(v_cache, e), SV_ERR_ALIGN);
  if (cache_dtype == SV_F8) {
    SV_REQUIRE(k_scale && v_scale, SV_ERR_NULL);
    SV_REQUIRE(is_aligned(k_scale, 4) && is_aligned(v_scale, 4), SV_ERR_ALIGN);
  }
  return SV_OK;
}

}  // namespace sv

extern "C" int sv_cache_write(const void* k, int64_t k_stride, const void* v, int64_t v_stride, const void* q_or_null,
                              int64_t q_stride, int Hq, void* q_out_or_null, int64_t q_out_stride,
                              const int32_t* t_offsets_or_null, int n_rows, const int32_t* lengths, const int32_t* pages,
                              int max_pages, int B, int P, int heads, int D, int dtype, const double* freq_or_null, int rot,
                              int layout, float amplitude, void* k_cache, void* v_cache, int cache_dtype,
                              float* k_scale_or_null, float* v_scale_or_null, int n_pages, int page,
                              uint32_t* flags_or_null, sv_stream_t stream) {
  using namespace sv;
  const int e = elem_bytes(dtype);
  SV_REQUIRE(e != 0 && (cache_dtype == dtype || cache_dtype == SV_F8), SV_ERR_DTYPE);
  const int status = check_rows(t_offsets_or_null, n_rows, B, P, max_pages, n_pages, heads, page, D);
  SV_REQUIRE(status == SV_OK, status);
  if (freq_or_null) {
    SV_REQUIRE(rot >= 2 && rot % 2 == 0 && rot <= D, SV_ERR_INVALID_ARG);
    SV_REQUIRE(layout == SV_ROPE_HALVES || layout == SV_ROPE_PAIRS, SV_ERR_INVALID_ARG);
    SV_REQUIRE(amplitude > 0.f && amplitude < INFINITY, SV_ERR_INVALID_ARG);
  }
  if (!t_offsets_or_null) n_rows = B * P;
  if (B == 0 || n_rows == 0) return SV_OK;
  SV_REQUIRE(k_stride >= (int64_t)heads * D && v_stride >= (int64_t)heads * D, SV_ERR_INVALID_ARG);
  SV_REQUIRE(k_stride < (1ll << 40) && v_stride < (1ll << 40), SV_ERR_TOO_LARGE);
  SV_REQUIRE((q_or_null != nullptr) == (q_out_or_null != nullptr), SV_ERR_NULL);
  if (q_or_null) {
    SV_REQUIRE(Hq >= 1 && q_stride >= (int64_t)Hq * D && q_out_stride >= (int64_t)Hq * D, SV_ERR_INVALID_ARG);
    SV_REQUIRE(Hq <= SV_HEADS_MAX && q_stride < (1ll << 40) && q_out_stride < (1ll << 40), SV_ERR_TOO_LARGE);
    SV_REQUIRE(q_or_null != q_out_or_null || q_stride == q_out_stride, SV_ERR_INVALID_ARG);
    SV_REQUIRE(is_aligned(q_or_null, e) && is_aligned(q_out_or_null, e), SV_ERR_ALIGN);
  }
  SV_REQUIRE(n_pages >= 1, SV_ERR_INVALID_ARG);
  SV_REQUIRE(k && v && lengths && pages, SV_ERR_NULL);
  const int cache = check_cache(k_cache, v_cache, k_scale_or_null, v_scale_or_null, cache_dtype, dtype);
  SV_REQUIRE(cache == SV_OK, cache);
  SV_REQUIRE(is_aligned(k, e) && is_aligned(v, e) && is_aligned(lengths, 4) && is_aligned(pages, 4) &&
                 is_aligned(t_offsets_or_null, 4) && is_aligned(freq_or_null, 8) && is_aligned(flags_or_null, 4),
             SV_ERR_ALIGN);
  if (!freq_or_null) rot = 0;
  const CacheArgs a{static_cast<const char*>(q_or_null), static_cast<const char*>(k), static_cast<const char*>(v),
                    static_cast<char*>(q_out_or_null), q_stride * e, k_stride * e, v_stride * e, q_out_stride * e,
                    q_or_null ? Hq : 0, tokens_of(n_rows), Rows{t_offsets_or_null, lengths, n_rows, B, P},
                    Pages{pages, max_pages, n_pages, heads, fast_div(page)}, freq_or_null, rope_shape(D, rot, dtype),
                    rope_shape(D, 0, dtype), (double)amplitude, static_cast<char*>(k_cache), static_cast<char*>(v_cache),
                    k_scale_or_null, v_scale_or_null, flags_or_null};
  const dim3 grid((n_rows + a.tokens - 1) / a.tokens);
  const size_t lds = (size_t)a.tokens * a.sh.pitch * sizeof(CosSin);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kRopeThreads), lds, as_stream(stream), a); };
  const bool pairs = rot > 0 && layout == SV_ROPE_PAIRS, f8 = cache_dtype == SV_F8;
  if (dtype == SV_F32) {
    if (f8) { if (pairs) go(cache_write_kernel<DT_F32, true, true>); else go(cache_write_kernel<DT_F32, false, true>); }
    else { if (pairs) go(cache_write_kernel<DT_F32, true, false>); else go(cache_write_kernel<DT_F32, false, false>); }
  } else {
    if (f8) { if (pairs) go(cache_write_kernel<DT_BF16, true, true>); else go(cache_write_kernel<DT_BF16, false, true>); }
    else { if (pairs) go(cache_write_kernel<DT_BF16, true, false>); else go(cache_write_kernel<DT_BF16, false, false>); }
  }
  return launch_status();
}

extern "C" int sv_cache_read(const void* k_cache, const void* v_cache, int cache_dtype, const float* k_scale_or_null,
                             const float* v_scale_or_null, int n_pages, int page, const int32_t* t_offsets_or_null, int n_rows,
                             const int32_t* start, const int32_t* pages, int max_pages, int B, int P, int heads, int D,
                             int dtype, void* k, int64_t k_stride, void* v, int64_t v_stride, uint32_t* flags_or_null,
                             sv_stream_t stream) {
  using namespace sv;
  const int e = elem_bytes(dtype);
  SV_REQUIRE(e != 0 && (cache_dtype == dtype || cache_dtype == SV_F8), SV_ERR_DTYPE);
  const int status = check_rows(t_offsets_or_null, n_rows, B, P, max_pages, n_pages, heads, page, D);
  SV_REQUIRE(status == SV_OK, status);
  if (!t_offsets_or_null) n_rows = B * P;
  if (B == 0 || n_rows == 0) return SV_OK;
  SV_REQUIRE(k_stride >= (int64_t)heads * D && v_stride >= (int64_t)heads * D, SV_ERR_INVALID_ARG);
  SV_REQUIRE(k_stride < (1ll << 40) && v_stride < (1ll << 40), SV_ERR_TOO_LARGE);
  SV_REQUIRE(n_pages >= 1, SV_ERR_INVALID_ARG);
  SV_REQUIRE(k && v && start && pages, SV_ERR_NULL);
  const int cache = check_cache(k_cache, v_cache, k_scale_or_null, v_scale_or_null, cache_dtype, dtype);
  SV_REQUIRE(cache == SV_OK, cache);
  SV_REQUIRE(is_aligned(k, e) && is_aligned(v, e) && is_aligned(start, 4) && is_aligned(pages, 4) &&
                 is_aligned(t_offsets_or_null, 4) && is_aligned(flags_or_null, 4),
             SV_ERR_ALIGN);
  const ReadArgs a{static_cast<char*>(k), static_cast<char*>(v), k_stride * e, v_stride * e, tokens_of(n_rows), D,
                   Rows{t_offsets_or_null, start, n_rows, B, P}, Pages{pages, max_pages, n_pages, heads, fast_div(page)},
                   static_cast<const char*>(k_cache), static_cast<const char*>(v_cache), k_scale_or_null, v_scale_or_null,
                   flags_or_null};
  const dim3 grid((n_rows + a.tokens - 1) / a.tokens);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kRopeThreads), 0, as_stream(stream), a); };
  if (dtype == SV_F32) {
    if (cache_dtype == SV_F8) go(cache_read_kernel<DT_F32, true>); else go(cache_read_kernel<DT_F32, false>);
  } else {
    if (cache_dtype == SV_F8) go(cache_read_kernel<DT_BF16, true>); else go(cache_read_kernel<DT_BF16, false>);
  }
  return launch_status();
}
