// sv_grad_norm, sv_clip_grad_norm: 2-norm over the elements of many tensors, and the tensors scaled by
// what the norm says.
//
// The tensors are cut into granules; a launch takes the addresses of up to kTensors of them by
// value.  A workgroup walks through granules one grid apart and leaves one fp64 sum of squares; one
// workgroup adds those up in a fixed order.  Bound by the bytes: the gradients are read twice (the
// factor is not known before all have been read) and written once.
#include "sv_device.hpp"
#include "sv_host.hpp"

namespace sv {

constexpr int kTensors = 120;           // tensors of one launch: 3.8 KB of kernel arguments
constexpr int kGranuleElems = 16384;
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
  constexpr int EPV = Elem<DT>::per_vec;
  double s = 0.0;
  for (int i = threadIdx.x; i < n / EPV; i += kNormThreads) {
    float f[EPV];
    unpack<DT>(load_vec(p, i), f);
#pragma unroll
    for (int j = 0; j < EPV; ++j) s = __builtin_fma((double)f[j], (double)f[j], s);
  }
  for (int i = n / EPV * EPV + threadIdx.x; i < n; i += kNormThreads) {
    const double x = (double)load_elem<DT>(p, i);
    s = __builtin_fma(x, x, s);
  }
  return s;
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

// One workgroup: norm, flag and factor from the partial sums.
__global__ __launch_bounds__(1024) void grad_norm_finish_kernel(const double* part, int n, float max_norm, float* norm,
                                                                uint32_t* flag, float* factor) {
  __shared__ BlockScratch sm;
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 1024) s += part[i];
  s = block_sum_f64(s, sm);
  if (threadIdx.x != 0) return;
  const float x = (float)sqrt(s);
  const bool fine = isfinite(x);
  *norm = x;
  if (flag) *flag = fine ? 0 : SV_FLAG_NONFINITE;
  *factor = fine ? (float)fmin(1.0, (double)max_norm / ((double)x + 1e-6)) : 1.f;
}

template <int DT, int DO>
__device__ __forceinline__ void scale_granule(const void* p, void* o, int n, float by) {
  constexpr int EPV = Elem<DT_BF16>::per_vec;          // 8 elements a step whatever the types
  for (int i = threadIdx.x; i < n / EPV; i += kNormThreads) {
    float f[EPV];
    if constexpr (DT == DT_BF16) {
      unpack<DT_BF16>(load_vec(p, i), f);
    } else {
      const u32x4 a = load_vec(p, 2 * i), c = load_vec(p, 2 * i + 1);
#pragma unroll
      for (int j = 0; j < 4; ++j) { f[j] = __uint_as_float(a[j]); f[4 + j] = __uint_as_float(c[j]); }
    }
#pragma unroll
    for (int j = 0; j < EPV; ++j) f[j] *= by;
    if constexpr (DO == DT_BF16) {
      u32x4 q;
#pragma unroll
      for (int j = 0; j < 4; ++j) q[j] = pack_bf16(f[2 * j], f[2 * j + 1]);
      reinterpret_cast<u32x4_row*>(o)[i] = q;
    } else {
      u32x4 q[2];
#pragma unroll
      for (int j = 0; j < EPV; ++j) q[j >> 2][j & 3] = __float_as_uint(f[j]);
      reinterpret_cast<u32x4_row*>(o)[2 * i] = q[0];
      reinterpret_cast<u32x4_row*>(o)[2 * i + 1] = q[1];
    }
  }
  for (int i = n / EPV * EPV + threadIdx.x; i < n; i += kNormThreads) {
    const float x = load_elem<DT>(p, i) * by;
    if constexpr (DO == DT_F32) static_cast<float*>(o)[i] = x;
    else static_cast<uint16_t*>(o)[i] = (uint16_t)pack_bf16(x, 0.f);
  }
}

__global__ __launch_bounds__(kNormThreads) void grad_scale_kernel(const TensorBatch b, const float* factor) {
  const float by = *factor;
  for (uint32_t g = blockIdx.x; g < b.granules; g += gridDim.x) {
    const TensorBatch::Entry& t = b.t[tensor_of(b, g)];
    if (by == 1.f && t.in == t.out) continue;
    const long long at = (long long)(g - t.first) * kGranuleElems;
    const int n = (int)min((long long)kGranuleElems, t.numel - at);
    const char* in = static_cast<const char*>(t.in) + at * (t.dtype == DT_F32 ? 4 : 2);
    char* out = static_cast<char*>(t.out) + at * (t.out_dtype == DT_F32 ? 4 : 2);
    if (t.dtype == DT_F32) {
      if (t.out_dtype == DT_F32) scale_granule<DT_F32, DT_F32>(in, out, n, by);
      else scale_granule<DT_F32, DT_BF16>(in, out, n, by);
    } else {
      if (t.out_dtype == DT_F32) scale_granule<DT_BF16, DT_F32>(in, out, n, by);
      else scale_granule<DT_BF16, DT_BF16>(in, out, n, by);
    }
  }
}

inline int batches(int n) { return n == 0 ? 1 : (n + kTensors - 1) / kTensors; }

// Tensors i0 .. of the lists, as one launch's arguments.
inline TensorBatch batch_of(int i0, int n, const void* const* grads, const int64_t* numel, const int* dtype,
                            void* const* out, const int* out_dtype) {
  TensorBatch b = {};
  for (int i = i0; i < n && i < i0 + kTensors; ++i) {
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
  long long granules = 0;
  for (int i = 0; i < n; ++i) {
    SV_REQUIRE((dtype[i] == SV_F32 || dtype[i] == SV_BF16) &&
                   (!out || out_dtype[i] == SV_F32 || out_dtype[i] == SV_BF16),
               SV_ERR_DTYPE);
    SV_REQUIRE(numel[i] >= 0, SV_ERR_INVALID_ARG);
    SV_REQUIRE(numel[i] <= (1LL << 44), SV_ERR_TOO_LARGE);
    granules += (numel[i] + kGranuleElems - 1) / kGranuleElems;
    SV_REQUIRE(granules <= 0x7fffffffLL, SV_ERR_TOO_LARGE);
    if (numel[i] == 0) continue;
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
  for (int i = 0; i < n; i += kTensors) {
    const TensorBatch b = batch_of(i, n, grads, numel, dtype, out, out_dtype);
    if (b.granules == 0) continue;
    const unsigned groups = b.granules < (uint32_t)kNormGroups ? b.granules : kNormGroups;
    hipLaunchKernelGGL(grad_norm_kernel, dim3(groups), dim3(kNormThreads), 0, st, b, part + parts);
    parts += (int)groups;
  }
  hipLaunchKernelGGL(grad_norm_finish_kernel, dim3(1), dim3(1024), 0, st, part, parts, max_norm, norm, flag, factor);
  for (int i = 0; out && i < n; i += kTensors) {
    const TensorBatch b = batch_of(i, n, grads, numel, dtype, out, out_dtype);
    if (b.granules == 0) continue;
    const unsigned groups = b.granules < 2u * kNormGroups ? b.granules : 2u * kNormGroups;
    hipLaunchKernelGGL(grad_scale_kernel, dim3(groups), dim3(kNormThreads), 0, st, b, factor);
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
