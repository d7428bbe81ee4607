// Clipped policy loss with a KL term, and its gradient, per token t and sub-model m:
//   D = logp - old,  r = e^D,  x = ref - logp
//   P = -min(r A, clamp(r, 1 - clip_low, 1 + clip_high) A)
//   K = e^x - x - 1                                (an estimate of KL(p || p_ref), >= 0)
//   L = P + beta K
//   dL/dlogp = (0 where the clamp decides the minimum, else -r A) - beta (e^x - 1)
// each times the token's weight: 1/N, 1/(B n_b) or 1 (N tokens count, n_b of them in
// sequence b).  Which side of a clipping bound a token is on decides between a
// gradient and none, so the comparison is made on D itself with the rounding of
// the subtraction kept (its exact value is D + e) against log(1 + clip_high) and
// log(1 - clip_low) in two fp32 words each: as exact as in 64 bits.  K of a small x
// comes from its series, not from a difference of numbers near 1.
//
// A block owns kPolicyTokens consecutive tokens: it finds each one's sequence,
// computes the weights once and goes through the sub-models.  How many tokens of
// a sequence count is known inside the block where the whole sequence is; for the
// (at most two) that cross the block's ends it comes from counts per chunk of
// tokens that a kernel before this one made.  Counts are integers and sums are
// added in a fixed order, so results do not depend on timing.
#include <climits>

#include "mls_device.cuh"
#include "mls_kernels.h"
#include "mls_vec.cuh"

namespace mls {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = kPolicyTokens / kThreads;

__device__ __forceinline__ bool counts(const PolicyParams& p, long long t) {
  const int y = p.y[t];
  return y >= 0 && y < p.V;
}

__device__ __forceinline__ int warp_sum_int(int v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sum over the block, valid in every thread; sh: kThreads / 32 values.
__device__ __forceinline__ int block_sum_int(int v, int* sh) {
  v = warp_sum_int(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  int s = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) s += sh[i];
  return s;
}

__device__ __forceinline__ double warp_sum_double(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Offset b of the sequences, within [0, T] whatever the caller's array holds.
__device__ __forceinline__ long long seq_at(const PolicyParams& p, int b) {
  const int v = p.seq_start[b];
  return v < 0 ? 0 : v > p.T ? p.T : v;
}

// The last of the sequences [lo, hi] that starts at or before t (lo if none does).
__device__ __forceinline__ int seq_of(const PolicyParams& p, long long t, int lo, int hi) {
  while (lo < hi) {
    const int mid = lo + ((hi - lo + 1) >> 1);
    if (p.seq_start[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Tokens of [lo, hi) that count; every thread of the block calls it with the same range.
__device__ int count_range(const PolicyParams& p, long long lo, long long hi, int* sh) {
  int n = 0;
  if (lo < hi) {
    const long long c0 = (lo + p.count_tokens - 1) / p.count_tokens, c1 = hi / p.count_tokens;
    if (c0 < c1) {  // whole chunks, and the two ends
      for (long long c = c0 + threadIdx.x; c < c1; c += kThreads) n += p.chunk_count[c];
      for (long long t = lo + threadIdx.x; t < c0 * p.count_tokens; t += kThreads) n += counts(p, t);
      for (long long t = c1 * p.count_tokens + threadIdx.x; t < hi; t += kThreads) n += counts(p, t);
    } else {
      for (long long t = lo + threadIdx.x; t < hi; t += kThreads) n += counts(p, t);
    }
  }
  return block_sum_int(n, sh);
}

__global__ void __launch_bounds__(kThreads) policy_count_kernel(const PolicyParams p) {
  __shared__ int sh[kThreads / 32];
  const long long t0 = static_cast<long long>(blockIdx.x) * p.count_tokens;
  const long long t1 = t0 + p.count_tokens < p.T ? t0 + p.count_tokens : p.T;
  // tokens outside every sequence do not count
  const long long lo = p.seq_start ? seq_at(p, 0) : 0, hi = p.seq_start ? seq_at(p, p.B) : p.T;
  int n = 0;
  for (long long t = t0 + threadIdx.x; t < t1; t += kThreads) n += t >= lo && t < hi && counts(p, t);
  n = block_sum_int(n, sh);
  if (threadIdx.x == 0) p.chunk_count[blockIdx.x] = n;
}

// e^x - 1 - x.  Below 1/2 its Taylor series (remainder under 2^-29 of it).
__device__ __forceinline__ float exp_excess(float x) {
  if (fabsf(x) < 0.5f) {
    float s = 1.f / 362880.f;
    s = fmaf(s, x, 1.f / 40320.f);
    s = fmaf(s, x, 1.f / 5040.f);
    s = fmaf(s, x, 1.f / 720.f);
    s = fmaf(s, x, 1.f / 120.f);
    s = fmaf(s, x, 1.f / 24.f);
    s = fmaf(s, x, 1.f / 6.f);
    s = fmaf(s, x, 0.5f);
    return x * x * s;
  }
  return expf(x) - 1.f - x;
}

// Sign of (d + e) - (hi + lo) for d + e an exact difference and hi + lo a bound, both
// with the second word under half a unit of the first's last place.
__device__ __forceinline__ float beyond(float d, float e, float hi, float lo) {
  return d == hi ? e - lo : (d - hi) + (e - lo);
}

struct Token {
  float policy, kl, grad;
  bool clipped;
};

__device__ __forceinline__ Token policy_token(const PolicyParams& p, float logp, float old, float ref,
                                              bool has_ref, float A) {
  const float d = logp - old;
  // the part of the exact difference that rounding d lost (Knuth's two-sum)
  const float back = d - logp;
  float e = (logp - (d - back)) - (old + back);
  if (!(fabsf(e) < INFINITY)) e = 0.f;  // d itself is infinite (or NaN): nothing was lost
  Token k;
  const bool over = A > 0.f && beyond(d, e, p.high[0], p.high[1]) > 0.f;
  const bool under = A < 0.f && beyond(d, e, p.low[0], p.low[1]) < 0.f;
  k.clipped = over || under;
  const float ratio = over ? p.ratio_high : under ? p.ratio_low : expf(d);
  k.policy = A == 0.f ? 0.f : -ratio * A;
  k.grad = k.clipped ? 0.f : k.policy;
  k.kl = 0.f;
  if (has_ref) {
    const float x = ref - logp;
    k.kl = exp_excess(x);
    if (p.beta != 0.f) k.grad = fmaf(-p.beta, fabsf(x) < 0.5f ? x + k.kl : expf(x) - 1.f, k.grad);
  }
  return k;
}

__global__ void __launch_bounds__(kThreads) policy_kernel(const __grid_constant__ PolicyParams p) {
  __shared__ int sh[kThreads / 32];
  __shared__ int inside[kPolicyTokens];  // counted tokens of the sequence that starts here
  __shared__ int ends[2];
  __shared__ double shd[kThreads / 32][3 * kMaxModels];
  const long long t0 = static_cast<long long>(blockIdx.x) * kPolicyTokens;
  const long long t1 = t0 + kPolicyTokens < p.T ? t0 + kPolicyTokens : p.T;
  const int B = p.B;

  if (p.agg == kAggSeq)
    for (int i = threadIdx.x; i < kPolicyTokens; i += kThreads) inside[i] = 0;
  if (p.seq_start && threadIdx.x < 2) ends[threadIdx.x] = seq_of(p, threadIdx.x ? t1 - 1 : t0, 0, B - 1);
  // The offsets have to be sorted and within [0, T].
  if (p.seq_start && blockIdx.x == 0)
    for (int b = threadIdx.x; b <= B; b += kThreads) {
      const int v = p.seq_start[b];
      if (v < 0 || v > p.T || (b > 0 && v < p.seq_start[b - 1])) atomicOr(p.status, kStatusBadSeq);
    }
  __syncthreads();
  const int b0 = p.seq_start ? ends[0] : 0, b1 = p.seq_start ? ends[1] : 0;

  // ---- each token's sequence, whether it counts, its advantage
  bool on[kPer];
  int seq[kPer];
  float A[kPer], weight[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const long long t = t0 + threadIdx.x + j * kThreads;
    on[j] = t < t1 && counts(p, t);
    seq[j] = 0;
    if (p.seq_start && on[j]) {
      seq[j] = seq_of(p, t, b0, b1);
      on[j] = t >= seq_at(p, seq[j]) && t < seq_at(p, seq[j] + 1);
    }
    A[j] = on[j] ? (p.adv_per_seq ? p.adv[seq[j]] : p.adv[t]) : 0.f;
    weight[j] = on[j] ? 1.f : 0.f;
  }

  // ---- weights
  if (p.agg == kAggToken) {
    int n = 0;
    if (p.chunks > 0) {
      for (int c = threadIdx.x; c < p.chunks; c += kThreads) n += p.chunk_count[c];
    } else {  // one block has all tokens
#pragma unroll
      for (int j = 0; j < kPer; ++j) n += on[j];
    }
    n = block_sum_int(n, sh);
    const float w = n > 0 ? 1.f / static_cast<float>(n) : 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) weight[j] *= w;
  } else if (p.agg == kAggSeq) {
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (on[j]) {
        const long long lo = seq_at(p, seq[j]);
        if (lo >= t0) atomicAdd(&inside[lo - t0], 1);
      }
    // the sequences that cross the block's ends
    int cross[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int b = q ? b1 : b0;
      const long long lo = seq_at(p, b), hi = seq_at(p, b + 1);
      cross[q] = 0;
      if (q == 1 && b0 == b1) cross[1] = cross[0];
      else if (lo < t0 || hi > t1) cross[q] = count_range(p, lo, hi, sh);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (on[j]) {
        const long long lo = seq_at(p, seq[j]), hi = seq_at(p, seq[j] + 1);
        const int n = lo >= t0 && hi <= t1 ? inside[lo - t0] : seq[j] == b0 ? cross[0] : cross[1];
        weight[j] = n > 0 ? static_cast<float>(1.0 / (static_cast<double>(B) * n)) : 0.f;
      }
  }

  // ---- loss and gradient of every sub-model
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int m = 0; m < p.M; ++m) {
    const long long row = static_cast<long long>(m) * p.T;
    const float gw = p.grad_scale * p.w[m];
    float sp = 0.f, sk = 0.f, sc = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const long long t = t0 + threadIdx.x + j * kThreads;
      if (t >= t1) continue;
      float L = 0.f, g = 0.f;
      if (on[j]) {
        const Token k = policy_token(p, p.logp[row + t], p.old_logp[row + t],
                                     p.ref_logp ? p.ref_logp[row + t] : 0.f, p.ref_logp != nullptr, A[j]);
        L = p.beta != 0.f ? fmaf(p.beta, k.kl, k.policy) : k.policy;  // beta 0: K is only reported
        g = k.grad * (weight[j] * gw);
        sp = fmaf(k.policy, weight[j], sp);
        sk = fmaf(k.kl, weight[j], sk);
        sc += k.clipped ? weight[j] : 0.f;
      }
      if (p.tok_loss) p.tok_loss[row + t] = L;
      if (p.dlogp) p.dlogp[row + t] = g;
    }
    const double a = warp_sum_double(sp), b = warp_sum_double(sk), c = warp_sum_double(sc);
    if (lane == 0) {
      shd[warp][3 * m] = a;
      shd[warp][3 * m + 1] = b;
      shd[warp][3 * m + 2] = c;
    }
  }
  __syncthreads();
  if (threadIdx.x < 3 * p.M) {
    double s = 0.0;
    for (int i = 0; i < kThreads / 32; ++i) s += shd[i][threadIdx.x];
    p.part[static_cast<long long>(blockIdx.x) * 3 * p.M + threadIdx.x] = s;
  }
}

// Block shares -> diag [3][M] and the loss.  Thread i adds shares i, i + threads, ...
// of one quantity; the threads are then added in order.
constexpr int kFinalThreads = 1024;

__global__ void __launch_bounds__(kFinalThreads) policy_final_kernel(const __grid_constant__ PolicyParams p, int blocks) {
  __shared__ double sh[kFinalThreads / 32];
  double loss = 0.0;
  for (int m = 0; m < p.M; ++m) {
    double v[3];
    for (int f = 0; f < 3; ++f) {
      double s = 0.0;
      for (int i = threadIdx.x; i < blocks; i += kFinalThreads) s += p.part[(static_cast<long long>(i) * p.M + m) * 3 + f];
      s = warp_sum_double(s);
      __syncthreads();
      if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
      __syncthreads();
      v[f] = 0.0;
      for (int i = 0; i < kFinalThreads / 32; ++i) v[f] += sh[i];
      if (p.diag && threadIdx.x == 0) p.diag[f * p.M + m] = static_cast<float>(v[f]);
    }
    loss += static_cast<double>(p.w[m]) * (p.beta != 0.f ? v[0] + static_cast<double>(p.beta) * v[1] : v[0]);
  }
  if (threadIdx.x == 0) *p.loss = static_cast<float>(loss);
}

}  // namespace

cudaError_t launch_policy(const PolicyParams& p, cudaStream_t s) {
  cudaError_t e;
  if (p.chunks > 0) {
    policy_count_kernel<<<p.chunks, kThreads, 0, s>>>(p);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
  }
  const int blocks = policy_blocks(p.T);
  policy_kernel<<<blocks, kThreads, 0, s>>>(p);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  policy_final_kernel<<<1, kFinalThreads, 0, s>>>(p, blocks);
  return cudaGetLastError();
}

}  // namespace mls
