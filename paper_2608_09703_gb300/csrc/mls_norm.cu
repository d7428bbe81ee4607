// Layer norm of the hidden states before a head, forward and backward.  Per token
// of d values:
//   mu = mean x,  r = 1 / sqrt(mean (x - mu)^2 + eps),  xh = (x - mu) r
//   y  = xh gain + bias
// Backward with g = dL/dy, h = g gain:
//   dL/dx = r (h - mean h - xh mean(h xh))
//   dL/dgain = sum over tokens of g xh,  dL/dbias = sum over tokens of g
// One warp owns a token; the variance is the mean of the squared deviations from
// the mean itself, so that a mean far from 0 costs no digits.  The column sums
// are taken in two steps: a block's rows into its own copy of the two rows of
// sums, then the copies, in order, so results do not depend on timing.
#include "mls_device.cuh"
#include "mls_kernels.h"
#include "mls_vec.cuh"

namespace mls {
namespace {

constexpr int kWarps = 4;

template <typename E>
__global__ void __launch_bounds__(32 * kWarps) norm_fwd_kernel(const NormParams p) {
  constexpr int N = Vec<E>::N;
  const long long t = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= p.T) return;
  const E* x = static_cast<const E*>(p.x) + t * p.d;
  const E* gain = static_cast<const E*>(p.gain);
  const E* bias = static_cast<const E*>(p.bias);
  E* y = static_cast<E*>(p.y) + t * p.d;
  const float inv_d = 1.0f / static_cast<float>(p.d);
  float s = 0.f, q = 0.f, f[N];
  for (int k = lane * N; k < p.d; k += 32 * N) {
    Vec<E>::unpack(ld16(x + k), f);
#pragma unroll
    for (int i = 0; i < N; ++i) s += f[i];
  }
  const float mu = warp_sum(s) * inv_d;
  for (int k = lane * N; k < p.d; k += 32 * N) {
    Vec<E>::unpack(ld16(x + k), f);
#pragma unroll
    for (int i = 0; i < N; ++i) q = fmaf(f[i] - mu, f[i] - mu, q);
  }
  const float r = 1.0f / sqrtf(warp_sum(q) * inv_d + p.eps);
  for (int k = lane * N; k < p.d; k += 32 * N) {
    float g[N], b[N];
    Vec<E>::unpack(ld16(x + k), f);
    if (gain) Vec<E>::unpack(ld16(gain + k), g);
    if (bias) Vec<E>::unpack(ld16(bias + k), b);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float xh = (f[i] - mu) * r;
      f[i] = fmaf(xh, gain ? g[i] : 1.f, bias ? b[i] : 0.f);
    }
    st16(y + k, Vec<E>::pack(f));
  }
  if (lane == 0) {
    if (p.mean) p.mean[t] = mu;
    if (p.rstd) p.rstd[t] = r;
  }
}

template <typename E>
__global__ void __launch_bounds__(32 * kWarps) norm_bwd_kernel(const NormParams p) {
  constexpr int N = Vec<E>::N;
  const long long t = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= p.T) return;
  const E* x = static_cast<const E*>(p.x) + t * p.d;
  const E* dy = static_cast<const E*>(p.dy) + t * p.d;
  const E* gain = static_cast<const E*>(p.gain);
  E* dx = static_cast<E*>(p.dx) + t * p.d;
  const float inv_d = 1.0f / static_cast<float>(p.d), mu = p.mean[t], r = p.rstd[t];
  float a = 0.f, b = 0.f, f[N], h[N], g[N];
  for (int k = lane * N; k < p.d; k += 32 * N) {
    Vec<E>::unpack(ld16(x + k), f);
    Vec<E>::unpack(ld16(dy + k), h);
    if (gain) Vec<E>::unpack(ld16(gain + k), g);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float hg = gain ? h[i] * g[i] : h[i];
      a += hg;
      b = fmaf(hg, (f[i] - mu) * r, b);
    }
  }
  a = warp_sum(a) * inv_d;
  b = warp_sum(b) * inv_d;
  for (int k = lane * N; k < p.d; k += 32 * N) {
    Vec<E>::unpack(ld16(x + k), f);
    Vec<E>::unpack(ld16(dy + k), h);
    if (gain) Vec<E>::unpack(ld16(gain + k), g);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float hg = gain ? h[i] * g[i] : h[i];
      f[i] = r * (hg - a - (f[i] - mu) * r * b);
    }
    st16(dx + k, Vec<E>::pack(f));
  }
}

// Column sums: a thread owns a column (x), a block every splits-th row (y).
constexpr int kColThreads = 128;

template <typename E>
__global__ void __launch_bounds__(kColThreads) norm_cols_kernel(const NormParams p) {
  const int c = blockIdx.x * kColThreads + threadIdx.x;
  if (c >= p.d) return;
  const E* x = static_cast<const E*>(p.x);
  const E* dy = static_cast<const E*>(p.dy);
  float dg = 0.f, db = 0.f;
  for (long long t = blockIdx.y; t < p.T; t += p.splits) {
    const float g = static_cast<float>(dy[t * p.d + c]);
    dg = fmaf(g, (static_cast<float>(x[t * p.d + c]) - p.mean[t]) * p.rstd[t], dg);
    db += g;
  }
  float* out = p.part + 2ll * p.d * blockIdx.y + c;
  out[0] = dg;
  out[p.d] = db;
}

__global__ void __launch_bounds__(kColThreads) norm_cols_sum_kernel(const NormParams p) {
  const int c = blockIdx.x * kColThreads + threadIdx.x;
  if (c >= p.d) return;
  float dg = 0.f, db = 0.f;
  for (int s = 0; s < p.splits; ++s) {
    dg += p.part[2ll * p.d * s + c];
    db += p.part[2ll * p.d * s + p.d + c];
  }
  if (p.dgain) p.dgain[c] = dg;
  if (p.dbias) p.dbias[c] = db;
}

unsigned blocks_of(long long n, int per) { return static_cast<unsigned>((n + per - 1) / per); }

}  // namespace

int norm_splits(long long T, int d, int sms) {
  const long long cols = (d + kColThreads - 1) / kColThreads;
  long long s = (8ll * sms + cols - 1) / cols;
  if (s > (T + 15) / 16) s = (T + 15) / 16;
  return s < 1 ? 1 : static_cast<int>(s);
}

cudaError_t launch_norm_fwd(const NormParams& p, bool fp32, cudaStream_t s) {
  if (p.T <= 0) return cudaSuccess;
  const unsigned grid = blocks_of(p.T, kWarps);
  if (fp32)
    norm_fwd_kernel<float><<<grid, 32 * kWarps, 0, s>>>(p);
  else
    norm_fwd_kernel<__nv_bfloat16><<<grid, 32 * kWarps, 0, s>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_norm_bwd(const NormParams& p, bool fp32, cudaStream_t s) {
  if (p.T <= 0) return cudaSuccess;
  cudaError_t e;
  if (p.dgain || p.dbias) {  // before dx, which may take dy's place
    const dim3 cols(blocks_of(p.d, kColThreads), p.splits);
    if (fp32)
      norm_cols_kernel<float><<<cols, kColThreads, 0, s>>>(p);
    else
      norm_cols_kernel<__nv_bfloat16><<<cols, kColThreads, 0, s>>>(p);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    norm_cols_sum_kernel<<<cols.x, kColThreads, 0, s>>>(p);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
  }
  const unsigned grid = blocks_of(p.T, kWarps);
  if (fp32)
    norm_bwd_kernel<float><<<grid, 32 * kWarps, 0, s>>>(p);
  else
    norm_bwd_kernel<__nv_bfloat16><<<grid, 32 * kWarps, 0, s>>>(p);
  return cudaGetLastError();
}

}  // namespace mls
