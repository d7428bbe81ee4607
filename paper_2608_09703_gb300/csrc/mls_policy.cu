// Clipped policy loss with a KL term, and its gradient, per token t and sub-model m:
//   D = logp - old,  r = e^D,  x = ref - logp
//   P = -min(r A, clamp(r, 1 - clip_low, 1 + clip_high) A)
//   K = e^x - x - 1                                (an estimate of KL(p || p_ref), >= 0)
//   L = P + beta K
//   dL/dlogp = (0 where the clamp decides the minimum, else -r A) - beta (e^x - 1)
// each times the token's weight: 1/N, 1/(B n_b) or 1 (N tokens count, n_b of them in
// sequence b).  Which side of a clipping bound a token is on decides between a
// gradient and none, so the comparison is made on D itself, and where D is near the
// bound with what rounding the subtraction lost (its exact value is D + e) and the
// bound, log(1 + clip_high) or log(1 - clip_low), in two fp32 words: right for every D that is
// not within 2^-47 of the bound.  K of a small x comes from its series, not from a difference
// of numbers near 1.
//
// A block owns 1024 consecutive tokens: it finds each one's sequence, computes the
// weights once and goes through the sub-models (or has one, see below).  How many
// tokens of a sequence count is known inside the block where the whole sequence is;
// for the (at most two) that cross the block's ends it comes from counts per chunk of
// tokens that a kernel before this one made.  Counts are integers and sums are
// added in a fixed order, so results do not depend on timing.
#include <climits>
#include <type_traits>

#include "mls_device.cuh"
#include "mls_kernels.h"
#include "mls_vec.cuh"

namespace mls {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = kPolicyTokens / kThreads;  // tokens of a thread
// Few tokens take one launch, a block of as many threads as it can have for each sub-model:
// 2000 tokens of 8 sequences, 1 / 2 / 4 sub-models 6.1 / 6.7 / 6.8 us; all sub-models in one
// block 6.7 / 8.3 / 11.0 (each is a chain of a load, an exponential and the sums); 1024 tokens
// a block and a second launch for the sums 7.9 / 8.9 / 11.4.
constexpr int kOneThreads = kPolicyOne / kPer;
// Blocks an SM holds of the main kernel, which its instructions bound: 63 registers with the
// next sub-model's inputs ahead.  4000001 tokens of 4 sub-models, KL term, sum: 71 us; 3 blocks
// 92; without the inputs ahead 79, that with 5 blocks 82.
constexpr int kResident = 4;

__device__ __forceinline__ bool counts(const PolicyParams& p, long long t) {
  const int y = p.y[t];
  return y >= 0 && y < p.V;
}

// Sum over the block of N threads, valid in every thread; sh: N / 32 values.
template <int N>
__device__ __forceinline__ int block_sum_int(int v, int* sh) {
  v = __reduce_add_sync(0xffffffffu, v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  int s = 0;
#pragma unroll
  for (int i = 0; i < N / 32; ++i) s += sh[i];
  return s;
}

// Starts of sequences that a block goes through one by one, in place of a search for
// each token.
constexpr int kFewSeqs = 32;

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

// The same by a whole warp, 32 candidates at a time: the search stands before
// everything else that the block does.
__device__ __forceinline__ int seq_of_warp(const PolicyParams& p, long long t, int hi, int lane) {
  int lo = 0;
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32;
    const long long c = lo + static_cast<long long>(lane + 1) * step;  // candidates lo + step, ...
    const unsigned below = __ballot_sync(0xffffffffu, c <= hi && p.seq_start[c] <= t);
    // sorted offsets give a run of ones from lane 0; of others, the run before the first zero
    const int k = __ffs(~below) == 0 ? 32 : __ffs(~below) - 1;
    lo += k * step;
    hi = lo + step - 1 < hi ? lo + step - 1 : hi;
  }
  return lo;
}

// Counted tokens among [lo, hi), this thread's share.
__device__ __forceinline__ int count_some(const PolicyParams& p, long long lo, long long hi) {
  int n = 0;
#pragma unroll 8
  for (long long t = lo + threadIdx.x; t < hi; t += kThreads) n += counts(p, t);
  return n;
}

// Counted tokens of sequence b if it crosses the block's ends, else 0: this thread's share.
__device__ __forceinline__ int count_crossing(const PolicyParams& p, int b, long long t0, long long t1) {
  long long lo = seq_at(p, b);
  const long long hi = seq_at(p, b + 1);
  if ((lo >= t0 && hi <= t1) || lo >= hi) return 0;
  int n = 0;
  if (p.chunks > 0) {
    const int sh = p.count_shift;
    const long long c0 = (lo + (1ll << sh) - 1) >> sh, c1 = hi >> sh;
    if (c0 < c1) {  // whole chunks, and the two ends
      for (long long c = c0 + threadIdx.x; c < c1; c += kThreads) n += p.chunk_count[c];
      n += count_some(p, lo, c0 << sh);
      lo = c1 << sh;
    }
  }
  return n + count_some(p, lo, hi);
}

// Counts of the chunks of tokens, and zeros up to a whole vector of four.
__global__ void __launch_bounds__(kThreads) policy_count_kernel(const __grid_constant__ PolicyParams p) {
  __shared__ int sh[kThreads / 32];
  chain_trigger();
  const long long t0 = static_cast<long long>(blockIdx.x) << p.count_shift, next = t0 + (1ll << p.count_shift);
  const long long t1 = next < p.T ? next : p.T;
  // tokens outside every sequence do not count
  const long long lo = p.seq_start ? seq_at(p, 0) : 0, hi = p.seq_start ? seq_at(p, p.B) : p.T;
  int n = 0;
#pragma unroll 4
  for (long long t = t0 + threadIdx.x; t < t1; t += kThreads) n += t >= lo && t < hi && counts(p, t);
  n = block_sum_int<kThreads>(n, sh);
  if (threadIdx.x == 0) p.chunk_count[blockIdx.x] = n;
  if (blockIdx.x == 0 && threadIdx.x < 4 && p.chunks + threadIdx.x < (p.chunks + 3) / 4 * 4)
    p.chunk_count[p.chunks + threadIdx.x] = 0;
}

// e^x - 1 - x and e^x - 1 for |x| < 1: with h = x / 2, whose series' remainder is under 2^-28.5 of
// it, e^x - 1 - x = 2 (e^h - 1 - h) + (e^h - 1)^2, of terms that are never negative.
constexpr float kSeries = 1.f;
__device__ __forceinline__ void exp_excess(float x, float& excess, float& minus_one) {
  const float h = 0.5f * x;
  float s = 1.f / 362880.f;
  s = fmaf(s, h, 1.f / 40320.f);
  s = fmaf(s, h, 1.f / 5040.f);
  s = fmaf(s, h, 1.f / 720.f);
  s = fmaf(s, h, 1.f / 120.f);
  s = fmaf(s, h, 1.f / 24.f);
  s = fmaf(s, h, 1.f / 6.f);
  s = fmaf(s, h, 0.5f);
  const float e = h * h * s, m = h + e;
  excess = fmaf(m, m, e + e);
  minus_one = x + excess;
}

// The loss of v[3 m], the sum of weight P, and v[3 m + 1], of weight K.  In two fp32 words: 64-bit
// arithmetic by one thread took a third of a microsecond a sub-model.
__device__ __forceinline__ float total_loss(const PolicyParams& p, const Pair* v) {
  Pair loss = {0.f, 0.f};
  for (int m = 0; m < p.M; ++m) {
    Pair a = v[3 * m];
    if (p.beta != 0.f) {
      const Pair k = pair_scaled(v[3 * m + 1], p.beta);
      pair_add(a, k.hi, k.lo);
    }
    a = pair_scaled(a, p.w[m]);
    pair_add(loss, a.hi, a.lo);
  }
  return pair_float(loss);
}

// One token's three inputs of a sub-model, for kPer tokens of a thread; i: the first.  kStep:
// distance of a thread's tokens; kFull: all of them are there.
struct Inputs {
  float logp[kPer], old[kPer], ref[kPer];
};
template <int kStep, bool kFull>
__device__ __forceinline__ void load_inputs(const PolicyParams& p, long long i, int left, Inputs& v) {
  const float *a = p.logp + i, *b = p.old_logp + i, *c = p.ref_logp ? p.ref_logp + i : a;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const bool in = kFull || j * kStep < left;
    v.logp[j] = in ? a[j * kStep] : 0.f;
    v.old[j] = in ? b[j * kStep] : 0.f;
    v.ref[j] = in ? c[j * kStep] : 0.f;
  }
}

// Sums of three values over the warp: lanes 8 f to 8 f + 7 return that of s[f].  Each of the
// first two exchanges halves the values that a lane still holds: 6 shuffles in place of 15.
__device__ __forceinline__ float warp_sum3(const float (&s)[3], int lane) {
  const bool up = lane & 16, odd = lane & 8;
  const float a = (up ? s[2] : s[0]) + __shfl_xor_sync(0xffffffffu, up ? s[0] : s[2], 16);
  const float b = (up ? 0.f : s[1]) + __shfl_xor_sync(0xffffffffu, up ? s[1] : 0.f, 16);
  float v = (odd ? b : a) + __shfl_xor_sync(0xffffffffu, odd ? a : b, 8);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The same in two words: all tokens' sums of a short batch, which no further sum evens out.
__device__ __forceinline__ Pair shfl_xor_pair(const Pair& a, int o) {
  return {__shfl_xor_sync(0xffffffffu, a.hi, o), __shfl_xor_sync(0xffffffffu, a.lo, o)};
}
__device__ __forceinline__ Pair warp_sum3_pair(const float (&s)[3], int lane) {
  const bool up = lane & 16, odd = lane & 8;
  Pair a = {up ? s[2] : s[0], 0.f}, b = {up ? 0.f : s[1], 0.f};
  pair_add(a, __shfl_xor_sync(0xffffffffu, up ? s[0] : s[2], 16), 0.f);
  pair_add(b, __shfl_xor_sync(0xffffffffu, up ? s[1] : 0.f, 16), 0.f);
  Pair v = odd ? b : a;
  const Pair other = shfl_xor_pair(odd ? a : b, 8);
  pair_add(v, other.hi, other.lo);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) {
    const Pair w = shfl_xor_pair(v, o);
    pair_add(v, w.hi, w.lo);
  }
  return v;
}

// A sub-model's loss and gradient of a thread's tokens kFrom to kTo - 1: adds to the sums s and writes.  The
// tokens side by side, without a branch but for what is rare; the ones that do not count
// are chosen away (a branch for each token and each of its cases: 92 in place of 79 us).
template <bool kRef, int kStep, bool kFull, int kFrom, int kTo>
__device__ __forceinline__ void policy_row(const PolicyParams& p, const Inputs& in, const bool (&on)[kPer],
                                           const float (&A)[kPer], const float (&weight)[kPer], float gw,
                                           long long i, int left, float (&s)[3]) {
  float *tok = p.tok_loss + i, *grad = p.dlogp + i;
  float d[kPer], past[kPer], kl[kPer], e1[kPer];
  bool near = false, large = false;
#pragma unroll
  for (int j = kFrom; j < kTo; ++j) {
    // The bound that this advantage meets: above for a gain, below for a loss.
    const bool up = A[j] > 0.f;
    d[j] = in.logp[j] - in.old[j];
    past[j] = d[j] - (up ? p.high[0] : p.low[0]);
    near |= fabsf(past[j]) <= (up ? p.high[2] : p.low[2]);  // as near as rounding can matter
    kl[j] = e1[j] = 0.f;
    if constexpr (kRef) {
      const float x = in.ref[j] - in.logp[j];
      exp_excess(x, kl[j], e1[j]);
      large |= fabsf(x) >= kSeries;
    }
  }
  if (near) {
#pragma unroll
    for (int j = kFrom; j < kTo; ++j) {
      const bool up = A[j] > 0.f;
      if (fabsf(past[j]) <= (up ? p.high[2] : p.low[2])) {
        // the part of the exact difference that rounding d lost (Knuth's two-sum), and the bound's second word
        const float back = d[j] - in.logp[j];
        const float e = (in.logp[j] - (d[j] - back)) - (in.old[j] + back);
        past[j] += (isfinite(d[j]) ? e : 0.f) - (up ? p.high[1] : p.low[1]);
      }
    }
  }
  if (kRef && large) {
#pragma unroll
    for (int j = kFrom; j < kTo; ++j) {
      const float x = in.ref[j] - in.logp[j];
      if (fabsf(x) >= kSeries) {
        e1[j] = expf(x) - 1.f;
        kl[j] = e1[j] - x;
      }
    }
  }
#pragma unroll
  for (int j = kFrom; j < kTo; ++j) {
    const bool up = A[j] > 0.f;
    const bool clipped = up ? past[j] > 0.f : A[j] < 0.f && past[j] < 0.f;
    const float ratio = expf(d[j]);
    float P = (clipped ? (up ? p.ratio_high : p.ratio_low) : ratio) * -A[j];
    P = A[j] == 0.f ? 0.f : P;
    float g = clipped ? 0.f : P, L = P, K = kl[j];
    if (kRef && p.beta != 0.f) {  // beta 0: K is only reported
      L = fmaf(p.beta, K, P);
      g = fmaf(-p.beta, e1[j], g);
    }
    L = on[j] ? L : 0.f;
    g = on[j] ? g * (weight[j] * gw) : 0.f;
    s[0] = fmaf(on[j] ? P : 0.f, weight[j], s[0]);
    if constexpr (kRef) s[1] = fmaf(on[j] ? K : 0.f, weight[j], s[1]);
    s[2] += clipped ? weight[j] : 0.f;
    if (kFull || (j * kStep < left && p.tok_loss)) tok[j * kStep] = L;
    if (kFull || (j * kStep < left && p.dlogp)) grad[j * kStep] = g;
  }
}

// kOne: one block has all tokens of a sub-model, counts them itself and writes the sums; the
// blocks are a cluster, whose first one adds up the loss.
template <bool kOne>
__global__ void __launch_bounds__(kOne ? kOneThreads : kThreads, kOne ? 1 : kResident) policy_kernel(const __grid_constant__ PolicyParams p) {
  constexpr int N = kOne ? kOneThreads : kThreads, kTokens = N * kPer;
  __shared__ int sh[N / 32], sh1[N / 32];
  __shared__ int inside[kTokens];  // counted tokens of the sequence that starts here
  __shared__ int ends[2];
  __shared__ int starts[kFewSeqs];
  __shared__ float advs[kFewSeqs];
  using Sum = std::conditional_t<kOne, Pair, float>;
  __shared__ Sum shf[N / 32][3 * kMaxModels];
  __shared__ __align__(8) Pair shq[3 * kMaxModels];
  // The block's sub-models [m0, m1): one where the grid has a row for each.
  const bool split = gridDim.y > 1;
  const int m0 = blockIdx.y, m1 = kOne || split ? m0 + 1 : p.M;
  const long long t0 = kOne ? 0 : static_cast<long long>(blockIdx.x) * kTokens;
  const long long t1 = t0 + kTokens < p.T ? t0 + kTokens : p.T;
  const int B = p.B, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // A warp's tokens follow one another where there are many (so that a prompt, tokens that do
  // not count, is left out by whole warps), else all warps have some.
  constexpr int kStep = kOne ? N : 32;
  const long long first = kOne ? t0 + threadIdx.x : t0 + warp * 32 * kPer + lane;
  const int left = static_cast<int>(t1 - first);  // this thread's token j: first + j kStep, if that is < left
  const bool full = t1 - t0 == kTokens && p.tok_loss && p.dlogp;
  if (!kOne) chain_trigger();
  if (kOne && split) cluster_arrive();

  // ---- what does not depend on the counts: the first sub-model's inputs, each
  // token's sequence, whether it counts, its advantage
  Inputs in;
  load_inputs<kStep, false>(p, m0 * p.T + first, left, in);
  bool on[kPer];
  float adv[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    on[j] = j * kStep < left && counts(p, first + j * kStep);
    adv[j] = !p.adv_per_seq && j * kStep < left ? p.adv[first + j * kStep] : 0.f;
  }
  if (p.agg == kAggSeq)
    for (int i = threadIdx.x; i < kTokens; i += N) inside[i] = 0;
  // The block's sequences [b0, b1], from all starts where they are few, else by search.
  const bool all = B <= kFewSeqs;
  int begin = 0, end = 0;
  if (p.seq_start) {
    begin = p.seq_start[0];
    end = p.seq_start[B];
    if (all) {
      if (threadIdx.x < kFewSeqs && threadIdx.x + 1 < B) starts[threadIdx.x] = p.seq_start[threadIdx.x + 1];
      if (threadIdx.x < kFewSeqs && threadIdx.x < B && p.adv_per_seq) advs[threadIdx.x] = p.adv[threadIdx.x];
    } else if (warp < 2) {
      const int b = seq_of_warp(p, warp ? t1 - 1 : t0, B - 1, lane);
      if (lane == 0) ends[warp] = b;
    }
  }
  // The offsets have to be sorted and within [0, T].  Every block looks at some: by one alone 200000
  // of them took 150 us.
  if (p.seq_start && blockIdx.y == 0) {
    auto look = [&](auto b) {
      const int v = p.seq_start[b];
      if (v < 0 || v > p.T || (b > 0 && v < p.seq_start[b - 1])) atomicOr(p.status, kStatusBadSeq);
    };
    if constexpr (kOne) {
      for (int b = threadIdx.x; b <= B; b += N) look(b);
    } else {  // 32 bits here: 82 us in place of 73 for 4000001 tokens
      for (long long b = static_cast<long long>(blockIdx.x) * N + threadIdx.x; b <= B; b += static_cast<long long>(gridDim.x) * N) look(b);
    }
  }
  __syncthreads();
  int b0 = 0, b1 = 0;
  if (p.seq_start && all) {
    for (int i = 0; i + 1 < B; ++i) {
      b0 += starts[i] <= t0;
      b1 += starts[i] < t1;
    }
  } else if (p.seq_start) {
    b0 = ends[0];
    b1 = ends[1];
  }
  int seq[kPer];
  float A[kPer], weight[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) seq[j] = b0;
  if (p.seq_start) {
    const int few = b1 - b0;
    if (few > 0 && few <= kFewSeqs) {  // each start of a sequence within the block, past b0's
      if (!all) {
        if (threadIdx.x < few) starts[threadIdx.x] = p.seq_start[b0 + 1 + threadIdx.x];
        __syncthreads();
      }
      for (int i = 0; i < few; ++i) {
        const int s = starts[all ? b0 + i : i];
#pragma unroll
        for (int j = 0; j < kPer; ++j) seq[j] += s <= first + j * kStep;
      }
    } else if (few > 0) {
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (on[j]) seq[j] = seq_of(p, first + j * kStep, b0, b1);
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const long long t = first + j * kStep;
      on[j] = on[j] && t >= begin && t < end;
    }
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    A[j] = on[j] ? (!p.adv_per_seq ? adv[j] : all ? advs[seq[j]] : p.adv[seq[j]]) : 0.f;
    weight[j] = on[j] ? 1.f : 0.f;
  }
  if (!kOne) chain_wait();  // the counts

  // ---- weights
  if (p.agg == kAggToken) {
    int n = 0;
    if constexpr (kOne) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) n += on[j];
    } else if (p.chunks == 0) {  // few tokens: each block counts them all
      n = count_some(p, p.seq_start ? seq_at(p, 0) : 0, p.seq_start ? seq_at(p, B) : p.T);
    } else {
      const int4* c = reinterpret_cast<const int4*>(p.chunk_count);
#pragma unroll 4
      for (int i = threadIdx.x; i < (p.chunks + 3) / 4; i += N) {
        const int4 v = c[i];
        n += (v.x + v.y) + (v.z + v.w);
      }
    }
    n = block_sum_int<N>(n, sh);
    const float w = n > 0 ? 1.f / static_cast<float>(n) : 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) weight[j] *= w;
  } else if (p.agg == kAggSeq) {
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (on[j]) {
        const long long lo = seq_at(p, seq[j]);
        if (lo >= t0 && lo < t1) atomicAdd(&inside[lo - t0], 1);
      }
    // the sequences that cross the block's ends
    int cross0 = 0, cross1 = 0;
    if constexpr (!kOne) {
      cross0 = count_crossing(p, b0, t0, t1);
      if (b1 != b0) cross1 = count_crossing(p, b1, t0, t1);
      cross0 = __reduce_add_sync(0xffffffffu, cross0);
      cross1 = __reduce_add_sync(0xffffffffu, cross1);
      if (lane == 0) {
        sh[warp] = cross0;
        sh1[warp] = cross1;
      }
      __syncthreads();
      cross0 = cross1 = 0;
#pragma unroll
      for (int i = 0; i < N / 32; ++i) {
        cross0 += sh[i];
        cross1 += sh1[i];
      }
      if (b1 == b0) cross1 = cross0;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (on[j]) {
        const long long lo = seq_at(p, seq[j]), hi = seq_at(p, seq[j] + 1);
        const int n = lo >= t0 && lo < t1 && hi <= t1 ? inside[lo - t0] : seq[j] == b0 ? cross0 : cross1;
        weight[j] = n > 0 ? 1.f / (static_cast<float>(B) * static_cast<float>(n)) : 0.f;
      }
  }

  // ---- loss and gradient of every sub-model
  bool some = false;
#pragma unroll
  for (int j = 0; j < kPer; ++j) some |= on[j];
  some = __any_sync(0xffffffffu, some);
  for (int m = m0; m < m1; ++m) {
    const long long i = static_cast<long long>(m) * p.T + first;
    const float gw = p.grad_scale * p.w[m];
    float s[3] = {0.f, 0.f, 0.f};
    Inputs next = in;
    if (some && m + 1 < m1) {
      if (full)
        load_inputs<kStep, true>(p, i + p.T, left, next);
      else
        load_inputs<kStep, false>(p, i + p.T, left, next);
    }
    if (!some) {
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (j * kStep < left) {
          if (p.tok_loss) p.tok_loss[i + j * kStep] = 0.f;
          if (p.dlogp) p.dlogp[i + j * kStep] = 0.f;
        }
    } else {
      auto row = [&](auto whole, auto from, auto to) {
        if (p.ref_logp)
          policy_row<true, kStep, whole.value, from.value, to.value>(p, in, on, A, weight, gw, i, left, s);
        else
          policy_row<false, kStep, whole.value, from.value, to.value>(p, in, on, A, weight, gw, i, left, s);
      };
      using std::integral_constant;
      constexpr integral_constant<int, 0> first_one;
      constexpr integral_constant<int, kPer> past_last;
      static_assert(kPer == 4, "the calls below");
      if constexpr (kOne) {  // a block of few tokens computes no more than it has
        row(std::false_type(), first_one, integral_constant<int, 1>());
        if (p.T > N) row(std::false_type(), integral_constant<int, 1>(), integral_constant<int, 2>());
        if (p.T > 2 * N) row(std::false_type(), integral_constant<int, 2>(), integral_constant<int, 3>());
        if (p.T > 3 * N) row(std::false_type(), integral_constant<int, 3>(), past_last);
      } else if (full) {
        row(std::true_type(), first_one, past_last);
      } else {
        row(std::false_type(), first_one, past_last);
      }
    }
    in = next;
    Sum sum = {};
    if constexpr (kOne) {
      if (some) sum = warp_sum3_pair(s, lane);
    } else {
      if (some) sum = warp_sum3(s, lane);
    }
    if (lane % 8 == 0 && lane < 24) shf[warp][3 * m + lane / 8] = sum;
  }
  __syncthreads();
  if (kOne && split) cluster_wait();  // the first block runs
  for (int q = 3 * m0 + warp; q < 3 * m1; q += N / 32) {  // a warp a quantity
    if constexpr (kOne) {
      static_assert(N == 32 * 32, "a lane for each warp");
      const Pair v = warp_sum_pair(shf[lane][q]);
      if (lane > 0) continue;
      if (split)
        store_remote(map_to_rank(smem_u32(&shq[q]), 0), v.hi, v.lo);
      else
        shq[q] = v;
      if (p.diag) p.diag[q % 3 * p.M + q / 3] = pair_float(v);
    } else {
      const float v = warp_sum(lane < N / 32 ? shf[lane][q] : 0.f);
      if (lane == 0) p.part[static_cast<long long>(q) * gridDim.x + blockIdx.x] = v;
    }
  }
  if constexpr (kOne) {
    if (split)
      cluster_sync();
    else
      __syncthreads();
    if (threadIdx.x == 0 && m0 == 0) *p.loss = total_loss(p, shq);
  }
}

// Block shares -> diag and the loss.  Each of the 3 M quantities has 32 / (3 M) warps;
// a lane adds its shares in two fp32 words (Pair): 64-bit additions by every thread
// took 25 us a sub-model, whatever the number of blocks.
constexpr int kFinalThreads = 1024, kFinalBatch = 16, kFinalFew = 2;

// Shares first, first + step, ... of `blocks`: kBatch loads at once, one latency for all.  An
// addition costs 30 cycles, of zeros behind the last share too (16 of them in place of 2 for
// 131072 tokens: 0.5 us).
template <int kBatch>
__device__ __forceinline__ void add_shares(Pair& a, const float* part, int first, int step, int blocks) {
  for (int i0 = first; i0 < blocks; i0 += kBatch * step) {
    float v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) v[u] = i0 + u * step < blocks ? part[i0 + u * step] : 0.f;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) pair_add(a, v[u], 0.f);
  }
}

__global__ void __launch_bounds__(kFinalThreads) policy_final_kernel(const __grid_constant__ PolicyParams p, int blocks) {
  __shared__ Pair sh[kFinalThreads / 32];
  __shared__ Pair total[3 * kMaxModels];
  const int nq = 3 * p.M, per = (kFinalThreads / 32) / nq, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int q = warp % nq, k = warp / nq;
  chain_wait();
  Pair a = {0.f, 0.f};
  if (k < per) {
    const float* part = p.part + static_cast<long long>(q) * blocks;
    if (blocks <= kFinalFew * per * 32)
      add_shares<kFinalFew>(a, part, k * 32 + lane, per * 32, blocks);
    else
      add_shares<kFinalBatch>(a, part, k * 32 + lane, per * 32, blocks);
  }
  a = warp_sum_pair(a);
  if (lane == 0) sh[warp] = a;
  __syncthreads();
  if (threadIdx.x < nq) {
    Pair b = sh[threadIdx.x];
    for (int i = 1; i < per; ++i) pair_add(b, sh[i * nq + threadIdx.x].hi, sh[i * nq + threadIdx.x].lo);
    total[threadIdx.x] = b;
    if (p.diag) p.diag[threadIdx.x % 3 * p.M + threadIdx.x / 3] = pair_float(b);
  }
  __syncthreads();
  if (threadIdx.x == 0) *p.loss = total_loss(p, total);
}

}  // namespace

cudaError_t launch_policy(const PolicyParams& p, cudaStream_t s) {
  const int blocks = policy_blocks(p.T);
  cudaError_t e;
  if (p.T <= kPolicyOne) {
    if (p.M == 1) {
      policy_kernel<true><<<1, kOneThreads, 0, s>>>(p);
      return cudaGetLastError();
    }
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.y = p.M;
    attr.val.clusterDim.x = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(1, p.M);
    cfg.blockDim = dim3(kOneThreads);
    cfg.stream = s;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if ((e = cudaLaunchKernelEx(&cfg, policy_kernel<true>, p)) != cudaSuccess) cudaGetLastError();
    return e;
  }
  // A block for each sub-model too where all fit at once, for the same reason: 40000 tokens, mean
  // over tokens, 4 sub-models 11.0 -> 8.3 us.  Beyond, a block finds sequences and weights once.
  const dim3 grid(blocks, static_cast<long long>(blocks) * p.M <= kResident * p.sms ? p.M : 1);
  if (p.chunks > 0) {
    policy_count_kernel<<<p.chunks, kThreads, 0, s>>>(p);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    if ((e = launch_chained(policy_kernel<false>, grid, dim3(kThreads), 0, s, p)) != cudaSuccess) return e;
  } else {
    policy_kernel<false><<<grid, kThreads, 0, s>>>(p);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
  }
  return launch_chained(policy_final_kernel, dim3(1), dim3(kFinalThreads), 0, s, p, blocks);
}

}  // namespace mls
