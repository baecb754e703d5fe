// sv_chunk_attention: what the rows and the scratch decide, the join of divided keys, the flags.
#include "attention.hpp"

namespace sv {

// Joins the parts of a row: a wavefront for each (new token, head).
template <int ET>
__global__ void __launch_bounds__(256) attention_join_kernel(AttnArgs a) {
  const int64_t at = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
  const int lane = threadIdx.x & (kWave - 1);
  const int hq = (int)(at % a.Hq);
  const int64_t bi = at / a.Hq;
  const int i = (int)(bi % a.rows.P), b = (int)(bi / a.rows.P);
  if (b >= a.rows.B) return;
  const int h = hq / a.group, rho = i * a.group + hq - h * a.group, tile = rho / a.tile_rows;
  const int item = (b * a.pages.heads + h) * a.tiles + tile;
  const int64_t part0 = (int64_t)item * a.splits * a.tile_rows + (rho - tile * a.tile_rows);
  // all asked for together: how many parts there are, whether the row is there, and maxima and sums of as many parts as there may be
  const int64_t p = part0 + (int64_t)min(lane, a.splits - 1) * a.tile_rows;
  float m = a.part_ml[2 * p], l = a.part_ml[2 * p + 1];
  const int parts = a.n_split[item];
  const Sequence s = sequence_of(a, b);
  if (i >= s.n || parts <= 1) return;
  m = lane < parts ? m : -INFINITY;
  l = lane < parts ? l : 0.f;
  const float top = wave_max_f32(m);
  const float f = m == top ? 1.f : exp2_fast(m - top);
  const double total = wave_sum_f64(lane < parts ? (double)l * f : 0.0);
  const bool out_of_pages = s.start + i >= s.cap;
  const bool any = top != -INFINITY || !(total == 0.0);
  const float inv = out_of_pages ? NAN : (any ? (float)(1.0 / total) : 0.f);
  if (a.lse && lane == 0)
    a.lse[(int64_t)(s.row0 + i) * a.Hq + hq] = out_of_pages ? NAN : (any ? (float)((top + log2(total)) * kLn2) : -INFINITY);
  char* to = a.out + (int64_t)(s.row0 + i) * a.out_stride;
  for (int col = 4 * lane; col < a.D; col += 4 * kWave) {
    f32x4 o{0.f, 0.f, 0.f, 0.f};
    typedef f32x4 vec __attribute__((aligned(4)));
    const float* from = a.part_o + part0 * a.D + col;
    for (int k0 = 0; k0 < parts; k0 += 8) {              // (eight parts under way together)
      f32x4 p[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k0 + k < parts) p[k] = *reinterpret_cast<const vec*>(from + (int64_t)(k0 + k) * a.tile_rows * a.D);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k0 + k < parts) o += p[k] * lane_f32(f, k0 + k);
    }
    o *= inv;
    if constexpr (ET == SV_F32) {
      typedef f32x4 vec __attribute__((aligned(4)));
      *reinterpret_cast<vec*>(to + ((int64_t)hq * a.D + col) * 4) = o;
    } else {
      typedef uint32_t vec __attribute__((ext_vector_type(2), aligned(2)));
      *reinterpret_cast<vec*>(to + ((int64_t)hq * a.D + col) * 2) = vec{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
    }
  }
}

// SV_FLAG_BAD_PAGE of every row that sees a key in no page: a wavefront for each new token.
__global__ void __launch_bounds__(256) attention_flags_kernel(AttnArgs a, uint32_t* flags) {
  const int64_t at = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
  const int lane = threadIdx.x & (kWave - 1), i = (int)(at % a.rows.P), b = (int)(at / a.rows.P);
  if (b >= a.rows.B) return;
  const Sequence s = sequence_of(a, b);
  if (i >= s.n) return;
  int lo, hi;
  keys_of(a, s, i, i, &lo, &hi);
  bool bad = s.start + i >= s.cap;
  if (hi > lo)
    for (int k = divide(lo, a.pages.page) + lane; k <= divide(hi - 1, a.pages.page); k += kWave) {
      const int p = a.pages.table[(int64_t)b * a.pages.max_pages + k];
      bad |= p < 0 || p >= a.pages.n_pages;
    }
  if (__ballot(bad) == 0) bad = false; else bad = true;
  if (lane == 0) flags[s.row0 + i] = bad ? SV_FLAG_BAD_PAGE : 0;
}

struct AttnPlan {
  int nt, tile_rows, tiles, splits;
  int64_t items;
  size_t bytes;
};

// How the rows of a call are laid out over workgroups: one block of up to 16, 32 or 48 rows to a wavefront, up to four of them.
inline AttnPlan attention_plan(int B, int P, int Hq, int heads, int D, int dtype, bool f8, int64_t max_tokens) {
  AttnPlan p{};
  const int64_t rows = (int64_t)P * (Hq / heads);
  const bool wide = dtype == SV_F32 || D > 128;             // (outputs of one block of rows fill a wavefront's registers)
  p.nt = wide || rows <= 16 ? 1 : 2;
  // (8-bit keys, converted once by one wavefront of 48 rows and not by two of 32, though 70 registers of it go to memory.  64 sequences of 8192 tokens, 4
  // heads to one, 48 rows and 32, us: 9 tokens of each, 128 columns, pages of 64 304 and 367, of 20 330 and 402; 64 columns 175 and 267, pages of 20 200 and
  // 318; 12 tokens, 128 columns 307 and 366, 64 columns 183 and 268.  Of 1 to 9 tokens over 2048 to 8192, where most sequences have
  // no more than 32 rows anyway: 128 columns 210 and 204, pages of 20 236 and 227, 64 columns 155 and 153; of 1 to 12 254 and 286, 163 and 206.
  // The worst found: 64 columns, 1 or 6 of 10 tokens, 152 and 128.  Keys of 16 bits do not leave the registers.)
  if (f8 && p.nt == 2 && rows > 32 && rows <= 48) p.nt = 3;
  p.tile_rows = 16 * p.nt * (rows <= 16 * p.nt ? 1 : (rows <= 32 * p.nt ? 2 : 4));
  const int64_t tiles = (rows + p.tile_rows - 1) / p.tile_rows;
  p.items = (int64_t)B * heads * tiles;
  p.tiles = (int)tiles;
  const int64_t most = (max_tokens + kMinSteps * kStep - 1) / (kMinSteps * kStep);
  int64_t splits = 4 * kTargetGroups / (p.items > 0 ? p.items : 1) + 1;
  splits = splits < most ? splits : most;
  // (what the parts take: each is written and read once, and 128 MB of them stay in the last-level cache)
  const int64_t room = kCacheBytes / (p.items * p.tile_rows * D * 4 > 0 ? p.items * p.tile_rows * D * 4 : 1);
  splits = splits < room ? splits : room;
  p.splits = (int)(splits < 1 ? 1 : (splits < kMaxSplits ? splits : kMaxSplits));
  p.bytes = 0;
  if (p.splits > 1)
    p.bytes = ws_round((size_t)p.items * 4) + ws_round((size_t)p.items * p.splits * p.tile_rows * 8) +
              ws_round((size_t)p.items * p.splits * p.tile_rows * D * 4);
  return p;
}

inline bool whole_tiles(int D, int page) { return (D == 64 || D == 128 || D == 256) && page % 16 == 0; }

}  // namespace sv

extern "C" size_t sv_chunk_attention_workspace_bytes(int B, int P, int Hq, int heads, int D, int dtype, int max_pages, int page) {
  using namespace sv;
  if (B < 1 || P < 1 || heads < 1 || Hq < heads || Hq % heads != 0 || Hq > SV_HEADS_MAX || D < 8 || D > SV_ATTENTION_HEAD_MAX || D % 8 != 0 ||
      elem_bytes(dtype) == 0 || max_pages < 1 || page < 1 || page > SV_PAGE_MAX || (long long)B * P > SV_TOKENS_MAX || (long long)B * P > kMaxRows / Hq)
    return 0;
  const size_t own = attention_plan(B, P, Hq, heads, D, dtype, false, (int64_t)max_pages * page).bytes;
  const size_t f8 = attention_plan(B, P, Hq, heads, D, dtype, true, (int64_t)max_pages * page).bytes;
  return own > f8 ? own : f8;
}

extern "C" int sv_chunk_attention(const void* q, int64_t q_stride, const int32_t* t_offsets_or_null, int n_rows,
                                  const int32_t* lengths, const int32_t* first_or_null, const int32_t* pages, int max_pages,
                                  int B, int P, int Hq, int heads, int D, int dtype, const void* k_cache,
                                  const void* v_cache, int cache_dtype, const float* k_scale_or_null,
                                  const float* v_scale_or_null, int n_pages, int page, float scale, int window, void* out,
                                  int64_t out_stride, float* lse_or_null, uint32_t* flags_or_null, void* ws_or_null,
                                  size_t ws_bytes, sv_stream_t stream) {
  using namespace sv;
  const int e = elem_bytes(dtype);
  SV_REQUIRE(e != 0 && (cache_dtype == dtype || cache_dtype == SV_F8), SV_ERR_DTYPE);
  const int status = check_rows(t_offsets_or_null, n_rows, B, P, max_pages, n_pages, heads, page, D);
  SV_REQUIRE(status == SV_OK, status);
  SV_REQUIRE(Hq >= heads && Hq % heads == 0 && D % 8 == 0 && window >= 0, SV_ERR_INVALID_ARG);
  SV_REQUIRE(scale > -INFINITY && scale < INFINITY, SV_ERR_INVALID_ARG);
  SV_REQUIRE(D <= SV_ATTENTION_HEAD_MAX && Hq <= SV_HEADS_MAX && (long long)B * P <= SV_TOKENS_MAX && (long long)B * P <= kMaxRows / Hq, SV_ERR_TOO_LARGE);
  if (!t_offsets_or_null) n_rows = B * P;
  if (B == 0 || n_rows == 0) return SV_OK;
  SV_REQUIRE(q_stride >= (int64_t)Hq * D && out_stride >= (int64_t)Hq * D, SV_ERR_INVALID_ARG);
  SV_REQUIRE(q_stride < (1ll << 40) && out_stride < (1ll << 40), SV_ERR_TOO_LARGE);
  SV_REQUIRE(n_pages >= 1 && q != out, SV_ERR_INVALID_ARG);
  SV_REQUIRE(q && out && lengths && pages && k_cache && v_cache, SV_ERR_NULL);
  const bool f8 = cache_dtype == SV_F8;
  SV_REQUIRE(!f8 || (k_scale_or_null && v_scale_or_null), SV_ERR_NULL);
  SV_REQUIRE(is_aligned(q, e) && is_aligned(out, e) && is_aligned(lengths, 4) && is_aligned(pages, 4) && is_aligned(t_offsets_or_null, 4) &&
                 is_aligned(first_or_null, 4) && is_aligned(lse_or_null, 4) && is_aligned(flags_or_null, 4) &&
                 is_aligned(k_cache, f8 ? 1 : e) && is_aligned(v_cache, f8 ? 1 : e) &&
                 (!f8 || (is_aligned(k_scale_or_null, 4) && is_aligned(v_scale_or_null, 4))),
             SV_ERR_ALIGN);
  const bool whole = whole_tiles(D, page);
  AttnPlan p = attention_plan(B, P, Hq, heads, D, dtype, f8, (int64_t)max_pages * page);
  if (!ws_or_null) p.splits = 1;
  else if (p.splits > 1) SV_REQUIRE(is_aligned(ws_or_null, kWsAlign) && ws_bytes >= p.bytes, SV_ERR_WORKSPACE);
  AttnArgs a{};
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.lse = lse_or_null;
  a.q_stride = q_stride * e;
  a.out_stride = out_stride * e;
  a.rows = Rows{t_offsets_or_null, lengths, n_rows, B, P};
  a.pages = Pages{pages, max_pages, n_pages, heads, fast_div(page)};
  a.first = first_or_null;
  a.Hq = Hq;
  a.group = Hq / heads;
  a.D = D;
  a.window = window;
  a.by_group = fast_div(a.group);
  a.zero = scale == 0.f && !f8;
  a.scale2 = a.zero ? 1.f : (float)((double)scale * kLog2e);
  a.k_cache = static_cast<const char*>(k_cache);
  a.v_cache = static_cast<const char*>(v_cache);
  a.k_scale = k_scale_or_null;
  a.v_scale = v_scale_or_null;
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.tile_rows = p.tile_rows;
  if (p.splits > 1) {
    char* w = static_cast<char*>(ws_or_null);
    a.n_split = reinterpret_cast<int*>(w);
    w += ws_round((size_t)p.items * 4);
    a.part_ml = reinterpret_cast<float*>(w);
    w += ws_round((size_t)p.items * p.splits * p.tile_rows * 8);
    a.part_o = reinterpret_cast<float*>(w);
  }
  // A launch holds 2^32 lanes: of more row blocks (which are not divided, so that no call needs scratch for them), as many sequences as one takes.
  // Those of one sequence fit, at most P Hq / 64 + heads.
  const int64_t each = (int64_t)heads * p.tiles * p.splits, most = 0xffffffffLL / (kAttnWaves * kWave) / each;
  for (int b = 0, n; b < B; b += n) {
    n = (int)(B - b < most ? B - b : most);
    AttnArgs s = a;
    s.rows.B = n;
    s.rows.start += b;
    s.pages.table += (int64_t)b * max_pages;
    if (s.first) s.first += b;
    if (s.rows.offsets) {
      s.rows.offsets += b;
    } else {
      s.q += (int64_t)b * P * s.q_stride;
      s.out += (int64_t)b * P * s.out_stride;
      if (s.lse) s.lse += (int64_t)b * P * Hq;
    }
    const AttnLaunch t{p.nt, p.nt == 2 && p.tile_rows == 128, whole, (unsigned)(n * each), as_stream(stream)};
    if (dtype == SV_F32) {
      if (f8) launch_attention_f32_f8(s, t); else launch_attention_f32(s, t);
    } else {
      if (f8) launch_attention_bf16_f8(s, t); else launch_attention_bf16(s, t);
    }
  }
  if (p.splits > 1) {
    const int64_t all = (int64_t)B * P * Hq;
    if (dtype == SV_F32)
      hipLaunchKernelGGL((attention_join_kernel<SV_F32>), dim3((unsigned)((all + 3) / 4)), dim3(256), 0, as_stream(stream), a);
    else
      hipLaunchKernelGGL((attention_join_kernel<SV_BF16>), dim3((unsigned)((all + 3) / 4)), dim3(256), 0, as_stream(stream), a);
  }
  if (flags_or_null)
    hipLaunchKernelGGL(attention_flags_kernel, dim3((unsigned)(((int64_t)B * P + 3) / 4)), dim3(256), 0, as_stream(stream), a, flags_or_null);
  return launch_status();
}
