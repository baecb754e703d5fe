// sv_grad_norm, sv_clip_grad_norm: 2-norm over the elements of many tensors, and the tensors scaled by
// what the norm says.
//
// The tensors are cut into granules; a launch takes the addresses of up to kTensors of them by
// value.  A workgroup walks through granules one grid apart and leaves one fp64 sum of squares.  Up to one launch of
// tensors, every workgroup of the second launch adds those up itself, in the same order; of more, one workgroup
// does in a launch between.  Bound by the bytes: the gradients are read twice (the factor is not known before
// all have been read) and written once.  The second reading goes backwards: what the first one read last is still in
// the last-level cache.  1.3e9 bf16 in 146 tensors: norm 445 us = 6.0 TB/s, scaling 1010 us = 5.3 TB/s read + write.
#include "sv_device.hpp"
#include "sv_host.hpp"

namespace sv {

constexpr int kTensors = 120;           // tensors of one launch: 3.8 KB of kernel arguments
constexpr int kGranuleElems = 8192;
constexpr int kNormGroups = 1024;       // workgroups of a launch at most
constexpr int kNormThreads = 256;

struct TensorBatch {
  struct Entry {
    const void* in;
    void* out;
    long long numel;
    uint32_t first;                     // granules of the tensors before it
    uint16_t dtype, out_dtype;
  } t[kTensors];
  int n;
  uint32_t granules;
};
static_assert(sizeof(TensorBatch) + 64 <= 4096, "kernel arguments");

// Tensor of a granule (uniform over the workgroup).
__device__ __forceinline__ int tensor_of(const TensorBatch& b, uint32_t granule) {
  int lo = 0, hi = b.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (b.t[mid].first <= granule) lo = mid; else hi = mid - 1;
  }
  return lo;
}

template <int DT>
__device__ __forceinline__ double squares(const void* p, int n) {
  constexpr int EPV = Elem<DT>::per_vec, U = 4;
  const int vecs = n / EPV, tid = threadIdx.x;
  double s[2] = {0.0, 0.0};
  auto add = [&](const u32x4& q) {
    float f[EPV];
    unpack<DT>(q, f);
#pragma unroll
    for (int j = 0; j < EPV; ++j) s[j & 1] = __builtin_fma((double)f[j], (double)f[j], s[j & 1]);
  };
  int i = tid;
  for (; i + (U - 1) * kNormThreads < vecs; i += U * kNormThreads) {
    u32x4 q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) q[u] = load_vec(p, i + u * kNormThreads);
#pragma unroll
    for (int u = 0; u < U; ++u) add(q[u]);
  }
  for (; i < vecs; i += kNormThreads) add(load_vec(p, i));
  for (int k = vecs * EPV + tid; k < n; k += kNormThreads) {
    const double x = (double)load_elem<DT>(p, k);
    s[0] = __builtin_fma(x, x, s[0]);
  }
  return s[0] + s[1];
}

__global__ __launch_bounds__(kNormThreads) void grad_norm_kernel(const TensorBatch b, double* part) {
  __shared__ BlockScratch sm;
  double s = 0.0;
  for (uint32_t g = blockIdx.x; g < b.granules; g += gridDim.x) {
    const TensorBatch::Entry& t = b.t[tensor_of(b, g)];
    const long long at = (long long)(g - t.first) * kGranuleElems;
    const int n = (int)min((long long)kGranuleElems, t.numel - at);
    if (t.dtype == DT_F32) s += squares<DT_F32>(static_cast<const float*>(t.in) + at, n);
    else s += squares<DT_BF16>(static_cast<const uint16_t*>(t.in) + at, n);
  }
  s = block_sum_f64(s, sm);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// What the partial sums say: the norm and, if `writes`, its outputs; the factor in every lane.
__device__ __forceinline__ float finish_norm(const double* part, int n, float max_norm, float* norm, uint32_t* flag,
                                             bool writes, BlockScratch& sm) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += kNormThreads) s += part[i];
  const float x = (float)sqrt(block_sum_f64(s, sm));
  const bool fine = isfinite(x);
  if (writes && threadIdx.x == 0) {
    *norm = x;
    if (flag) *flag = fine ? 0 : SV_FLAG_NONFINITE;
  }
  return fine ? (float)fmin(1.0, (double)max_norm / ((double)x + 1e-6)) : 1.f;
}

__global__ __launch_bounds__(kNormThreads) void grad_norm_finish_kernel(const double* part, int n, float max_norm,
                                                                        float* norm, uint32_t* flag, float* factor) {
  __shared__ BlockScratch sm;
  const float by = finish_norm(part, n, max_norm, norm, flag, true, sm);
  if (threadIdx.x == 0) *factor = by;
}

// ONCE: the results are more than the last-level cache keeps for a later reader, and are written past it.
template <int DT, int DO, bool ONCE>
__device__ __forceinline__ void scale_granule(const void* p, void* o, int n, float by) {
  constexpr int kIn = DT == DT_BF16 ? 1 : 2, U = 4;    // 8 elements a step whatever the types
  const int steps = n / 8, tid = threadIdx.x;
  auto load = [&](int i, u32x4 (&q)[kIn]) {
#pragma unroll
    for (int k = 0; k < kIn; ++k) q[k] = load_vec(p, kIn * i + k);
  };
  auto store = [&](int i, const u32x4 (&q)[kIn]) {
    float f[8];
    if constexpr (DT == DT_BF16) {
      unpack<DT_BF16>(q[0], f);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(q[j >> 2][j & 3]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= by;
    u32x4 r[2];
    auto put = [&](const u32x4& v, int at) {
      u32x4_row* to = reinterpret_cast<u32x4_row*>(o) + at;
      if constexpr (ONCE) __builtin_nontemporal_store(v, to);
      else *to = v;
    };
    if constexpr (DO == DT_BF16) {
#pragma unroll
      for (int j = 0; j < 4; ++j) r[0][j] = pack_bf16(f[2 * j], f[2 * j + 1]);
      put(r[0], i);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j >> 2][j & 3] = __float_as_uint(f[j]);
      put(r[0], 2 * i);
      put(r[1], 2 * i + 1);
    }
  };
  int i = tid;
  for (; i + (U - 1) * kNormThreads < steps; i += U * kNormThreads) {
    u32x4 q[U][kIn];
#pragma unroll
    for (int u = 0; u < U; ++u) load(i + u * kNormThreads, q[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) store(i + u * kNormThreads, q[u]);
  }
  for (; i < steps; i += kNormThreads) {
    u32x4 q[kIn];
    load(i, q);
    store(i, q);
  }
  for (int k = steps * 8 + tid; k < n; k += kNormThreads) {
    const float x = load_elem<DT>(p, k) * by;
    if constexpr (DO == DT_F32) static_cast<float*>(o)[k] = x;
    else static_cast<uint16_t*>(o)[k] = (uint16_t)pack_bf16(x, 0.f);
  }
}

struct Finish {
  const double* part;                 // the partial sums, if this launch is to add them up
  int n;
  float max_norm;
  float* norm;
  uint32_t* flag;
  const float* factor;                // else: the factor
};
static_assert(sizeof(TensorBatch) + sizeof(Finish) <= 4096, "kernel arguments");

template <bool ONCE>
__global__ __launch_bounds__(kNormThreads) void grad_scale_kernel(const TensorBatch b, const Finish f) {
  __shared__ BlockScratch sm;
  const float by = f.part ? finish_norm(f.part, f.n, f.max_norm, f.norm, f.flag, blockIdx.x == 0, sm) : *f.factor;
  for (uint32_t k = blockIdx.x; k < b.granules; k += gridDim.x) {
    const uint32_t g = b.granules - 1 - k;
    const TensorBatch::Entry& t = b.t[tensor_of(b, g)];
    if (by == 1.f && t.in == t.out) continue;
    const long long at = (long long)(g - t.first) * kGranuleElems;
    const int n = (int)min((long long)kGranuleElems, t.numel - at);
    const char* in = static_cast<const char*>(t.in) + at * (t.dtype == DT_F32 ? 4 : 2);
    char* out = static_cast<char*>(t.out) + at * (t.out_dtype == DT_F32 ? 4 : 2);
    if (t.dtype == DT_F32) {
      if (t.out_dtype == DT_F32) scale_granule<DT_F32, DT_F32, ONCE>(in, out, n, by);
      else scale_granule<DT_F32, DT_BF16, ONCE>(in, out, n, by);
    } else {
      if (t.out_dtype == DT_F32) scale_granule<DT_BF16, DT_F32, ONCE>(in, out, n, by);
      else scale_granule<DT_BF16, DT_BF16, ONCE>(in, out, n, by);
    }
  }
}

inline int batches(int n) { return n == 0 ? 1 : (n - 1) / kTensors + 1; }

// Batch k of the lists' tensors, as one launch's arguments.
inline TensorBatch batch_of(int k, int n, const void* const* grads, const int64_t* numel, const int* dtype,
                            void* const* out, const int* out_dtype) {
  TensorBatch b = {};
  const int first = k * kTensors, here = n - first < kTensors ? n - first : kTensors;
  for (int i = first; i - first < here; ++i) {
    if (numel[i] == 0) continue;
    b.t[b.n++] = {grads[i], out ? out[i] : nullptr, numel[i], b.granules, (uint16_t)dtype[i],
                  (uint16_t)(out ? out_dtype[i] : 0)};
    b.granules += (uint32_t)((numel[i] + kGranuleElems - 1) / kGranuleElems);
  }
  return b;
}

}  // namespace sv

namespace {
int norm_and_scale(int n, const void* const* grads, const int64_t* numel, const int* dtype, float max_norm,
                   void* const* out, const int* out_dtype, float* norm, uint32_t* flag, void* ws, size_t ws_bytes,
                   sv_stream_t stream) {
  using namespace sv;
  SV_REQUIRE(n >= 0, SV_ERR_INVALID_ARG);
  SV_REQUIRE(norm && (n == 0 || (grads && numel && dtype)), SV_ERR_NULL);
  long long granules = 0, bytes = 0;
  for (int i = 0; i < n; ++i) {
    SV_REQUIRE((dtype[i] == SV_F32 || dtype[i] == SV_BF16) &&
                   (!out || out_dtype[i] == SV_F32 || out_dtype[i] == SV_BF16),
               SV_ERR_DTYPE);
    SV_REQUIRE(numel[i] >= 0, SV_ERR_INVALID_ARG);
    SV_REQUIRE(numel[i] <= (1LL << 44), SV_ERR_TOO_LARGE);
    granules += (numel[i] + kGranuleElems - 1) / kGranuleElems;
    SV_REQUIRE(granules <= 0x7fffffffLL, SV_ERR_TOO_LARGE);
    if (numel[i] == 0) continue;
    bytes += numel[i] * (elem_bytes(dtype[i]) + (out ? elem_bytes(out_dtype[i]) : 0));
    SV_REQUIRE(grads[i] && (!out || out[i]), SV_ERR_NULL);
    SV_REQUIRE(is_aligned(grads[i], elem_bytes(dtype[i])) && (!out || is_aligned(out[i], elem_bytes(out_dtype[i]))),
               SV_ERR_ALIGN);
    SV_REQUIRE(!out || out[i] != grads[i] || out_dtype[i] == dtype[i], SV_ERR_INVALID_ARG);
  }
  SV_REQUIRE(is_aligned(norm, 4) && is_aligned(flag, 4), SV_ERR_ALIGN);
  SV_REQUIRE(ws && is_aligned(ws, kWsAlign) && ws_bytes >= sv_grad_norm_workspace_bytes(n), SV_ERR_WORKSPACE);
  float* factor = static_cast<float*>(ws);
  double* part = reinterpret_cast<double*>(static_cast<char*>(ws) + kWsAlign);
  hipStream_t st = as_stream(stream);
  int parts = 0;
  for (int k = 0; k < batches(n); ++k) {
    const TensorBatch b = batch_of(k, n, grads, numel, dtype, out, out_dtype);
    if (b.granules == 0) continue;
    const unsigned groups = b.granules < (uint32_t)kNormGroups ? b.granules : kNormGroups;
    hipLaunchKernelGGL(grad_norm_kernel, dim3(groups), dim3(kNormThreads), 0, st, b, part + parts);
    parts += (int)groups;
  }
  const bool apart = !out || parts == 0 || n > kTensors;
  if (apart)
    hipLaunchKernelGGL(grad_norm_finish_kernel, dim3(1), dim3(kNormThreads), 0, st, part, parts, max_norm, norm, flag, factor);
  for (int k = batches(n) - 1; out && k >= 0; --k) {
    const TensorBatch b = batch_of(k, n, grads, numel, dtype, out, out_dtype);
    if (b.granules == 0) continue;
    const unsigned groups = b.granules < 2u * kNormGroups ? b.granules : 2u * kNormGroups;
    const Finish f = {apart ? nullptr : part, parts, max_norm, norm, flag, factor};
    if (bytes > kCacheBytes) hipLaunchKernelGGL(grad_scale_kernel<true>, dim3(groups), dim3(kNormThreads), 0, st, b, f);
    else hipLaunchKernelGGL(grad_scale_kernel<false>, dim3(groups), dim3(kNormThreads), 0, st, b, f);
  }
  return launch_status();
}
}  // namespace

extern "C" size_t sv_grad_norm_workspace_bytes(int n) {
  if (n < 0) return 0;
  return sv::kWsAlign + (size_t)sv::batches(n) * sv::kNormGroups * 8;
}

extern "C" int sv_grad_norm(int n, const void* const* grads, const int64_t* numel, const int* dtype, float* norm,
                            uint32_t* flag_or_null, void* ws, size_t ws_bytes, sv_stream_t stream) {
  return norm_and_scale(n, grads, numel, dtype, 1.f, nullptr, nullptr, norm, flag_or_null, ws, ws_bytes, stream);
}

extern "C" int sv_clip_grad_norm(int n, const void* const* grads, const int64_t* numel, const int* dtype,
                                 float max_norm, void* const* out, const int* out_dtype, float* norm,
                                 uint32_t* flag_or_null, void* ws, size_t ws_bytes, sv_stream_t stream) {
  SV_REQUIRE(max_norm > 0.f, SV_ERR_INVALID_ARG);        // (false for NaN)
  SV_REQUIRE(n == 0 || (out && out_dtype), SV_ERR_NULL);
  return norm_and_scale(n, grads, numel, dtype, max_norm, out, out_dtype, norm, flag_or_null, ws, ws_bytes, stream);
}
