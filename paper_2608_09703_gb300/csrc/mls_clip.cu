// Global gradient norm over many tensors, and clipping in place:
//   n = sqrt(sum over all tensors of g^2),  c = min(1, max_norm / (n + 1e-6)),  g *= c
// A call's tensors come as a table in the kernels' parameters (kClipTable of them
// a launch), cut into chunks of kClipChunk values that persistent blocks take in
// turn.  Squares are summed in fp32 over the 32 values that a thread holds of a
// chunk, in two fp32 words (Pair) over a block, and in 64 bits from there on.  Where
// such a sum leaves the range in which fp32 squares are exact to rounding (a square
// that overflowed, or squares so small that some vanished) those 32 values are taken
// times a power of two, into sums of their own (Blue's method), so the norm is right
// from the smallest to the largest representable gradient at about the same speed.
// The blocks' shares are added in a fixed order: results do not depend on timing.
#include "mls_device.cuh"
#include "mls_kernels.h"
#include "mls_vec.cuh"

namespace mls {
namespace {

constexpr int kThreads = 256;

// The tensor of chunk c: the last one whose first chunk is not past c.
template <int kCap>
__device__ __forceinline__ int tensor_of(const ClipParams<kCap>& p, int c) {
  int lo = 0, hi = p.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (p.t[mid].chunk0 <= c) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// What a thread has summed: squares as they are, of values times 2^90, of values times 2^-80.
struct Squares {
  Pair plain, tiny, huge;
};
constexpr float kUp = 0x1p90f, kDown = 0x1p-80f;

template <int n>
__device__ __forceinline__ float scaled_squares(const float (&f)[n], float scale) {
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < n; ++i) s[i & 3] = fmaf(f[i] * scale, f[i] * scale, s[i & 3]);
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// Adds the squares of a thread's values of a chunk, see above.
template <int n>
__device__ __forceinline__ void add_squares(Squares& acc, const float (&f)[n]) {
  const float a = scaled_squares(f, 1.f);
  if (a >= 0x1p-80f && a <= 0x1p90f)
    pair_add(acc.plain, a, 0.f);
  else if (a < 0x1p-80f)
    pair_add(acc.tiny, scaled_squares(f, kUp), 0.f);  // at most 2^100 each
  else
    pair_add(acc.huge, scaled_squares(f, kDown), 0.f);  // at most 2^101 each; infinite or NaN stays
}

// Chunk `local` of a tensor: whole vectors of 16 bytes where there are any, single
// values at its end.  A tensor that starts off a 16-byte boundary has `head`
// values before its first vector, which go with chunk 0.
template <typename E>
__device__ __forceinline__ void chunk_squares(const E* g, const ClipTensor& t, int local, Squares& acc) {
  constexpr int N = Vec<E>::N, kV = kClipChunk / kThreads / N;
  const long long first = t.head + static_cast<long long>(local) * kClipChunk;
  float f[kV * N];
  if (first + kClipChunk <= t.numel) {  // every load issued before the first is used
    uint4 u[kV];
#pragma unroll
    for (int v = 0; v < kV; ++v) u[v] = ld16(g + first + (v * kThreads + static_cast<int>(threadIdx.x)) * N);
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      float w[N];
      Vec<E>::unpack(u[v], w);
#pragma unroll
      for (int i = 0; i < N; ++i) f[v * N + i] = w[i];
    }
  } else {
#pragma unroll
    for (int v = 0; v < kV; ++v) {
      const long long e = first + (v * kThreads + static_cast<int>(threadIdx.x)) * N;
      float w[N];
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = 0.f;
      if (e + N <= t.numel) {
        Vec<E>::unpack(ld16(g + e), w);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (e + i < t.numel) w[i] = static_cast<float>(g[e + i]);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) f[v * N + i] = w[i];
    }
  }
  add_squares(acc, f);
  if (local == 0 && static_cast<int>(threadIdx.x) < t.head) {
    const float h[1] = {static_cast<float>(g[threadIdx.x])};
    add_squares(acc, h);
  }
}

template <int kCap>
__global__ void __launch_bounds__(kThreads, kClipNormBlocks) clip_norm_kernel(const __grid_constant__ ClipParams<kCap> p) {
  chain_trigger();
  __shared__ Pair sh[kThreads / 32];
  __shared__ double shr[kThreads / 32];
  __shared__ bool has[kThreads / 32];
  Squares acc = {};
  for (int c = blockIdx.x; c < p.chunks; c += gridDim.x) {
    const ClipTensor& t = p.t[tensor_of(p, c)];
    if (t.fp32)
      chunk_squares(static_cast<const float*>(t.g), t, c - t.chunk0, acc);
    else
      chunk_squares(static_cast<const __nv_bfloat16*>(t.g), t, c - t.chunk0, acc);
  }
  const Pair s = warp_sum_pair(acc.plain);
  // what the other two hold, rarely anything; also where one is NaN
  const bool some = acc.tiny.hi != 0.f || acc.huge.hi != 0.f;
  const bool warp_has = __any_sync(0xffffffffu, some);
  double r = 0.0;
  if (warp_has) {
    if (some) r = pair_value(acc.tiny) * 0x1p-180 + pair_value(acc.huge) * 0x1p160;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) r += __shfl_down_sync(0xffffffffu, r, o);
  }
  if ((threadIdx.x & 31) == 0) {
    sh[threadIdx.x >> 5] = s;
    shr[threadIdx.x >> 5] = r;
    has[threadIdx.x >> 5] = warp_has;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    Pair a = sh[0];
    for (int i = 1; i < kThreads / 32; ++i) pair_add(a, sh[i].hi, sh[i].lo);
    double total = pair_value(a);
    for (int i = 0; i < kThreads / 32; ++i)
      if (has[i]) total += shr[i];
    p.part[p.part0 + blockIdx.x] = total;
  }
}

template <typename E>
__device__ __forceinline__ void chunk_scale(E* g, const ClipTensor& t, int local, float coef) {
  constexpr int N = Vec<E>::N, kV = kClipChunk / kThreads / N;
  const long long first = t.head + static_cast<long long>(local) * kClipChunk;
  uint4 u[kV];
#pragma unroll
  for (int v = 0; v < kV; ++v) {
    const long long e = first + (v * kThreads + static_cast<int>(threadIdx.x)) * N;
    if (e + N <= t.numel) u[v] = ld16(g + e);
  }
#pragma unroll
  for (int v = 0; v < kV; ++v) {
    const long long e = first + (v * kThreads + static_cast<int>(threadIdx.x)) * N;
    if (e + N <= t.numel) {
      float w[N];
      Vec<E>::unpack(u[v], w);
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] *= coef;
      st16(g + e, Vec<E>::pack(w));
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (e + i < t.numel) g[e + i] = static_cast<E>(static_cast<float>(g[e + i]) * coef);
    }
  }
  if (local == 0 && static_cast<int>(threadIdx.x) < t.head)
    g[threadIdx.x] = static_cast<E>(static_cast<float>(g[threadIdx.x]) * coef);
}

// a / (hi + lo) rounded once, of a finite quotient: one Newton step on the fp32 one.
__device__ __forceinline__ float quotient(float a, float hi, float lo) {
  const float q = a / hi;
  return q + fmaf(-q, lo, fmaf(-q, hi, a)) / hi;
}

// The norm of a sum of squares a and the factor for it, each rounded once.  The root and the
// quotient are fp32's, of a times a power of 4 in [1, 4), each with a Newton step that takes up what
// they lost: in 64 bits they took half a microsecond.
__device__ __forceinline__ float norm_of(double a, float max_norm, float& coef) {
  const int e = ((__double2hiint(a) >> 20) & 0x7ff) - 1023;
  if (e == 1024 || a == 0.0) {
    // NaN stays (every gradient becomes NaN); an infinite norm gives 0, as the formula says
    const float n = static_cast<float>(a);
    coef = isinf(max_norm) ? 1.f : a == 0.0 ? fminf(1.f, max_norm / 1e-6f) : isinf(n) ? 0.f : n;
    return n;
  }
  const int h = e >> 1;  // a = m 4^h
  const double m = __hiloint2double(__double2hiint(a) - 2 * h * (1 << 20), __double2loint(a));
  const float r = sqrtf(static_cast<float>(m));
  const float rest = static_cast<float>(fma(-static_cast<double>(r), static_cast<double>(r), m)) * 0.5f / r;
  const float norm = ldexpf(r + rest, h);
  float ratio;
  if (h > 64) {  // a norm past fp32's largest value still has its factor; 1e-6 is nothing to it
    ratio = ldexpf(quotient(max_norm, r, rest), -h);
  } else {
    constexpr double kEps = 1e-6;
    const float n = ldexpf(r, h);
    Pair d = {n, ldexpf(rest, h)};
    pair_add(d, static_cast<float>(kEps), static_cast<float>(kEps - static_cast<float>(kEps)));
    ratio = max_norm / d.hi < 2.f ? quotient(max_norm, d.hi, d.lo) : 2.f;
  }
  coef = isinf(max_norm) || ratio >= 1.f ? 1.f : ratio;
  return norm;
}

// Every block adds all shares of the norm itself, in the same order: its first warp,
// since 64-bit additions of all warps would only queue for the SM's two units.
template <int kCap>
__global__ void __launch_bounds__(kThreads, kClipScaleBlocks) clip_scale_kernel(const __grid_constant__ ClipParams<kCap> p) {
  __shared__ float sh_coef;
  chain_trigger();
  chain_wait();
  if (threadIdx.x < 32) {
    double a = 0.0;
#pragma unroll 8
    for (int i = threadIdx.x; i < p.nparts; i += 32) a += p.part[i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a += __shfl_down_sync(0xffffffffu, a, o);
    if (threadIdx.x == 0) {
      float c;
      const float norm = norm_of(a, p.max_norm, c);
      sh_coef = c;
      if (p.stats && blockIdx.x == 0) {
        p.stats[0] = norm;
        p.stats[1] = c;
      }
    }
  }
  __syncthreads();
  const float coef = sh_coef;
  if (coef == 1.f) return;  // nothing to change
  for (int i = blockIdx.x; i < p.chunks; i += gridDim.x) {
    const int c = p.chunks - 1 - i;  // the values read last are the likeliest in L2
    const ClipTensor& t = p.t[tensor_of(p, c)];
    if (t.fp32)
      chunk_scale(static_cast<float*>(t.g), t, c - t.chunk0, coef);
    else
      chunk_scale(static_cast<__nv_bfloat16*>(t.g), t, c - t.chunk0, coef);
  }
}

}  // namespace

template <int kCap>
cudaError_t launch_clip_norm(const ClipParams<kCap>& p, int grid, cudaStream_t s) {
  clip_norm_kernel<kCap><<<grid, kThreads, 0, s>>>(p);
  return cudaGetLastError();
}
template <int kCap>
cudaError_t launch_clip_scale(const ClipParams<kCap>& p, int grid, cudaStream_t s) {
  return launch_chained(clip_scale_kernel<kCap>, dim3(grid), dim3(kThreads), 0, s, p);
}
template cudaError_t launch_clip_norm(const ClipParams<kClipTable>&, int, cudaStream_t);
template cudaError_t launch_clip_scale(const ClipParams<kClipTable>&, int, cudaStream_t);
template cudaError_t launch_clip_norm(const ClipParams<kClipFew>&, int, cudaStream_t);
template cudaError_t launch_clip_scale(const ClipParams<kClipFew>&, int, cudaStream_t);

}  // namespace mls
