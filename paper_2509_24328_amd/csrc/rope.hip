// sv_rope_frequencies, sv_rope: rotary positions of queries or keys outside a cache, and of their gradients.
#include "rope.hpp"

namespace sv {

struct RopeArgs {
  const char* x;
  char* out;
  const int32_t* positions;
  const double* freq;
  int64_t x_stride, out_stride;      // bytes from token to token
  int n, H, head_bytes, tokens;      // tokens of a workgroup
  RopeShape sh;
  double amplitude, sign;
  bool in_place;
};

// A workgroup turns the heads of `tokens` tokens: their angles once, in LDS, then a head for every eight lanes.  What bounds it is the
// memory: each column is read once and written once (16384 tokens x 32 heads of 128 bf16 columns 58 us, 4.6 TB/s; 9 x 14 of 64 3.5 us, a chain of
// positions, frequencies, sines and one head).
template <int DT, bool PAIRS>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(RopeArgs a) {
  extern __shared__ CosSin cs[];                       // [tokens][pitch]
  const int t0 = blockIdx.x * a.tokens, nt = min(a.tokens, a.n - t0), half = a.sh.half;
  for (int k = threadIdx.x; k < nt * half; k += kRopeThreads) {
    const int t = k / half;
    cs[t * a.sh.pitch + angle_at<Elem<DT>::per_vec>(k - t * half)] = cos_sin((double)a.positions[t0 + t] * a.freq[k - t * half] * a.sign, a.amplitude);
  }
  __syncthreads();
  const int lane = threadIdx.x % kRopeLanes;
  for (int k = threadIdx.x / kRopeLanes; k < nt * a.H; k += kRopeGroups) {
    const int t = k / a.H, h = k - t * a.H;
    if (a.positions[t0 + t] < 0) continue;
    const char* row = a.x + (t0 + t) * a.x_stride + (int64_t)h * a.head_bytes;
    char* to = a.out + (t0 + t) * a.out_stride + (int64_t)h * a.head_bytes;
    turn_head<DT, PAIRS>(row, a.sh, cs + t * a.sh.pitch, lane, a.in_place,
                         [&](int at, int n, const float (&f)[Elem<DT>::per_vec]) { store_some<DT>(to, at, n, f); });
  }
}

__global__ void rope_frequencies_kernel(int half, double log_base, int scaling, double factor, double low, double high,
                                        double length, double* freq) {
  const int j = blockIdx.x * blockDim.x + threadIdx.x;
  if (j >= half) return;
  double f = exp(-((double)j / half) * log_base);
  if (scaling == SV_ROPE_LINEAR) f /= factor;
  if (scaling == SV_ROPE_PARTS) {
    const double turns = length * f / (2.0 * 3.14159265358979323846);
    const double keep = fmin(fmax((turns - low) / (high - low), 0.0), 1.0);
    f = f / factor * (1.0 - keep) + f * keep;
  }
  freq[j] = f;
}

}  // namespace sv

extern "C" int sv_rope_frequencies(int rot, double base, int scaling, double factor, double low, double high, int length,
                                   double* freq, sv_stream_t stream) {
  using namespace sv;
  SV_REQUIRE(rot >= 2 && rot % 2 == 0 && base > 1.0 && base < INFINITY, SV_ERR_INVALID_ARG);
  SV_REQUIRE(scaling >= SV_ROPE_PLAIN && scaling <= SV_ROPE_PARTS, SV_ERR_INVALID_ARG);
  if (scaling != SV_ROPE_PLAIN) SV_REQUIRE(factor > 0.0 && factor < INFINITY, SV_ERR_INVALID_ARG);
  if (scaling == SV_ROPE_PARTS) SV_REQUIRE(low >= 0.0 && high > low && high < INFINITY && length >= 1, SV_ERR_INVALID_ARG);
  SV_REQUIRE(rot <= SV_HEAD_MAX, SV_ERR_TOO_LARGE);
  SV_REQUIRE(freq, SV_ERR_NULL);
  SV_REQUIRE(is_aligned(freq, 8), SV_ERR_ALIGN);
  double log_base = __builtin_log(base);
  if (scaling == SV_ROPE_NTK && rot > 2) log_base += __builtin_log(factor) * (rot / (rot - 2.0));
  hipLaunchKernelGGL(rope_frequencies_kernel, dim3((rot / 2 + 63) / 64), dim3(64), 0, as_stream(stream), rot / 2, log_base, scaling,
                     factor, low, high, (double)length, freq);
  return launch_status();
}

extern "C" int sv_rope(const void* x, int64_t x_stride, const int32_t* positions, int n, int H, int D, int dtype,
                       const double* freq, int rot, int layout, float amplitude, int inverse, void* out,
                       int64_t out_stride, sv_stream_t stream) {
  using namespace sv;
  const int e = elem_bytes(dtype);
  SV_REQUIRE(e != 0, SV_ERR_DTYPE);
  SV_REQUIRE(n >= 0 && H >= 1 && D >= 1 && rot >= 2 && rot % 2 == 0 && rot <= D, SV_ERR_INVALID_ARG);
  SV_REQUIRE(layout == SV_ROPE_HALVES || layout == SV_ROPE_PAIRS, SV_ERR_INVALID_ARG);
  SV_REQUIRE(amplitude > 0.f && amplitude < INFINITY, SV_ERR_INVALID_ARG);
  SV_REQUIRE(D <= SV_HEAD_MAX && H <= SV_HEADS_MAX && n <= SV_TOKENS_MAX, SV_ERR_TOO_LARGE);   // (64 threads to a row, 2^32 to a launch)
  SV_REQUIRE(x_stride >= (int64_t)H * D && out_stride >= (int64_t)H * D, SV_ERR_INVALID_ARG);
  SV_REQUIRE(x_stride < (1ll << 40) && out_stride < (1ll << 40), SV_ERR_TOO_LARGE);
  SV_REQUIRE(x != out || x_stride == out_stride, SV_ERR_INVALID_ARG);
  if (n == 0) return SV_OK;
  SV_REQUIRE(x && positions && freq && out, SV_ERR_NULL);
  SV_REQUIRE(is_aligned(x, e) && is_aligned(out, e) && is_aligned(positions, 4) && is_aligned(freq, 8), SV_ERR_ALIGN);
  RopeArgs a{static_cast<const char*>(x), static_cast<char*>(out), positions, freq, x_stride * e, out_stride * e, n, H, D * e,
             // four tokens share a workgroup's start where every compute unit has several workgroups anyway
             n >= 4096 ? 4 : 1, rope_shape(D, rot, dtype), (double)amplitude, inverse ? -1.0 : 1.0, x == out};
  const dim3 grid((n + a.tokens - 1) / a.tokens);
  const size_t lds = (size_t)a.tokens * a.sh.pitch * sizeof(CosSin);
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kRopeThreads), lds, as_stream(stream), a); };
  if (dtype == SV_F32) {
    if (layout == SV_ROPE_PAIRS) go(rope_kernel<DT_F32, true>); else go(rope_kernel<DT_F32, false>);
  } else {
    if (layout == SV_ROPE_PAIRS) go(rope_kernel<DT_BF16, true>); else go(rope_kernel<DT_BF16, false>);
  }
  return launch_status();
}
