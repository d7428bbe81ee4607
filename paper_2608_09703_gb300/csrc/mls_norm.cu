// Layer norm of the hidden states before a head, forward and backward.  Per token
// of d values:
//   mu = mean x,  r = 1 / sqrt(mean (x - mu)^2 + eps),  xh = (x - mu) r
//   y  = xh gain + bias
// Backward with g = dL/dy, h = g gain:
//   dL/dx = r (h - mean h - xh mean(h xh))
//   dL/dgain = sum over tokens of g xh,  dL/dbias = sum over tokens of g
// Bound by HBM: forward x and y, backward x, g and dx, each moved once.  The variance
// is the mean of the squared deviations from the mean itself, so that a mean far
// from 0 costs the digits of its own rounding only, not those of its square.
//   forward   a row stays in the registers of its 1 to 16 warps, at most 8 16-byte
//             vectors a lane;
//   backward  persistent blocks of 16 warps, W of them to a row, which copy rows ahead
//             into shared memory and keep their columns' sums of g xh and g in
//             registers over all rows of the block (the widest rows: split over a cluster of
//             two CTAs).  The blocks' sums are added in order by a second
//             kernel, so results do not depend on timing;
//   wider rows are read again from L2 instead, one warp a row, their sums in two words.
#include "mls_device.cuh"
#include "mls_kernels.h"
#include "mls_vec.cuh"

namespace mls {
namespace {

__device__ __forceinline__ void group_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// ------------------------------------------------------------------ forward
// V vectors a lane, W warps a row: vector j of warp w's lane l is number (j W + w) 32 + l.
// Rows of at most 8 or 16 vectors (V = W = 1) take L lanes each, 32 / L of them a warp.
template <int W>
constexpr int kFwdGroups = W < 4 ? 4 / W : 1;  // groups of W warps a block

template <int L>
__device__ __forceinline__ float lane_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <int W, int L>
__device__ __forceinline__ float row_sum(float v, float* sh, int id, int w) {
  v = lane_sum<L>(v);
  if constexpr (W > 1) {
    if ((threadIdx.x & 31) == 0) sh[w] = v;
    group_sync(id, 32 * W);
    v = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) v += sh[i];
  }
  return v;
}

template <typename E, int V, int W, int L>
__global__ void __launch_bounds__(32 * W * kFwdGroups<W>) norm_fwd_kernel(const NormParams p) {
  constexpr int N = Vec<E>::N, N2 = Vec2<E>::N, kRows = 32 / L;
  __shared__ float sh[kFwdGroups<W>][2][W];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & (L - 1), group = warp / W, w = warp % W;
  const long long t0 = (static_cast<long long>(blockIdx.x) * kFwdGroups<W> + group) * kRows;
  if (t0 >= p.T) return;  // whole groups
  const long long t = t0 + (threadIdx.x & 31) / L;
  const int d = kRows == 1 || t < p.T ? p.d : 0;  // a row past the last one has no values
  const E* x = static_cast<const E*>(p.x) + t * p.d;
  E* y = static_cast<E*>(p.y) + t * p.d;
  uint4 u[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int k = ((j * W + w) * L + lane) * N;
    u[j] = k < d ? ld16(x + k) : make_uint4(0u, 0u, 0u, 0u);
  }
  const float inv_d = 1.0f / static_cast<float>(p.d);
  F2 f[V][N2];
  F2 s = 0, q = 0;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    Vec2<E>::unpack(u[j], f[j]);
#pragma unroll
    for (int i = 0; i < N2; ++i) s = f2_add(s, f[j][i]);
  }
  const float mu = row_sum<W, L>(f2_sum(s), sh[group][0], 1 + group, w) * inv_d;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const bool in = ((j * W + w) * L + lane) * N < d;
#pragma unroll
    for (int i = 0; i < N2; ++i) {
      f[j][i] = f2_add(f[j][i], f2(in ? -mu : 0.f));
      q = f2_fma(f[j][i], f[j][i], q);
    }
  }
  const float r = 1.0f / sqrtf(row_sum<W, L>(f2_sum(q), sh[group][1], 1 + group, w) * inv_d + p.eps);
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int k = ((j * W + w) * L + lane) * N;
    if (k < d) {
      // no gain: ones, no bias: zeros
      const uint32_t one = Vec2<E>::kOne;
      F2 g[N2], b[N2];
      Vec2<E>::unpack(p.gain ? ld16(static_cast<const E*>(p.gain) + k) : make_uint4(one, one, one, one), g);
      Vec2<E>::unpack(p.bias ? ld16(static_cast<const E*>(p.bias) + k) : make_uint4(0u, 0u, 0u, 0u), b);
#pragma unroll
      for (int i = 0; i < N2; ++i) f[j][i] = f2_fma(f2_mul(f[j][i], f2(r)), g[i], b[i]);
      st16(y + k, Vec2<E>::pack(f[j]));
    }
  }
  if (w == 0 && lane == 0 && d > 0 && p.mean) {
    p.mean[t] = mu;
    p.rstd[t] = r;
  }
}

// ------------------------------------------------------------------ backward
constexpr int kBwdWarps = 16;

// 16 bytes from global to shared memory without a register; a thread's copies since its
// last commit form a group, and it waits until at most N of its groups are left.
__device__ __forceinline__ void copy16_async(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// S rows of every lane's own vectors in shared memory, S - 1 of them being copied there
// (cp.async: a lane waits for and reads its own copies only, so no barrier is needed):
// with a row ahead in registers alone, 32 KB were in flight on an SM, and 65536 x
// 4096 bf16 values took 372 us.
// C = 2: the widest rows are split over a cluster of two CTAs, half the columns each, which
// exchange their sums of each row through shared memory.
template <typename E, int V, int W, int S, int L, int C>
__global__ void __launch_bounds__(32 * kBwdWarps, 1) norm_bwd_kernel(const NormParams p) {
  constexpr int N = Vec<E>::N, N2 = Vec2<E>::N, kGroups = kBwdWarps / W, kThreads = 32 * kBwdWarps;
  constexpr int kRows = 32 / L;
  static_assert(C == 1 || (W == kBwdWarps && L == 32), "a split row takes all warps of both CTAs");
  const int rank = C == 1 ? 0 : static_cast<int>(cluster_ctarank());
  // the CTA's columns [from, to): halves of whole vectors of all lanes of a warp
  const int half = C == 1 ? 0 : (p.d / 2 + 32 * N - 1) / (32 * N) * (32 * N);
  const int from = rank * half, to = C == 1 || rank == 1 ? p.d : half;
  const unsigned block = blockIdx.x / C, blocks = gridDim.x / C;
  extern __shared__ __align__(16) uint4 ring[];  // [S][x, g][V][kThreads], after the loop the sums [2][d]
  __shared__ float2 sh[2][C * kBwdWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & (L - 1), part = (threadIdx.x & 31) / L;
  const int group = warp / W, w = warp % W;
  const E* gain = static_cast<const E*>(p.gain);
  const float inv_d = 1.0f / static_cast<float>(p.d);
  const uint32_t one = Vec2<E>::kOne;
  uint4 gv[V];  // the gain; ones without one
  F2 dg[V][N2], db[V][N2];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int k = from + ((j * W + w) * L + lane) * N;
    gv[j] = gain && k < to ? ld16(gain + k) : make_uint4(one, one, one, one);
#pragma unroll
    for (int i = 0; i < N2; ++i) dg[j][i] = db[j][i] = 0;
  }
  const long long step = static_cast<long long>(blocks) * kGroups * kRows;
  long long t0 = (static_cast<long long>(block) * kGroups + group) * kRows;  // the warp's first row
  long long t = t0 + part;
  const uint32_t mine = smem_u32(ring) + threadIdx.x * 16;
  auto fetch = [&](long long row, int slot) {
    if (row < p.T) {
      const E* x = static_cast<const E*>(p.x) + row * p.d;
      const E* g = static_cast<const E*>(p.dy) + row * p.d;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int k = from + ((j * W + w) * L + lane) * N;
        if (k < to) {
          copy16_async(mine + (slot * 2 * V + j) * kThreads * 16, x + k);
          copy16_async(mine + (slot * 2 * V + V + j) * kThreads * 16, g + k);
        }
      }
    }
    copy_commit();
  };
#pragma unroll
  for (int q = 0; q < S - 1; ++q) fetch(t + q * step, q);
  if constexpr (C > 1) cluster_sync();  // both CTAs run before either writes to the other
  float mu = 0.f, r = 0.f;
  if (t < p.T) {
    mu = p.mean[t];
    r = p.rstd[t];
  }
  int slot = 0;
  for (int it = 0; t0 < p.T; t0 += step, t += step, it ^= 1) {
    const int d = kRows == 1 || t < p.T ? to : 0;  // a row past the last one has no values
    fetch(t + (S - 1) * step, slot == 0 ? S - 1 : slot - 1);  // the slot read in the round before
    copy_wait<S - 1>();
    const F2 nmu = f2(-mu), r2 = f2(r);
    if (t + step < p.T) {  // the next row's
      mu = p.mean[t + step];
      r = p.rstd[t + step];
    }
    // xh and h stay in registers; where those hold 64 sums they are formed again from the ring
    constexpr bool kAgain = V * N2 > 8;
    F2 a2 = 0, b2 = 0, xh[kAgain ? 1 : V][N2], h[kAgain ? 1 : V][N2];
    auto form = [&](int j, F2 (&x)[N2], F2 (&hh)[N2], F2 (&g)[N2]) {
      F2 gn[N2];
      Vec2<E>::unpack(ring[(slot * 2 * V + j) * kThreads + threadIdx.x], x);
      Vec2<E>::unpack(ring[(slot * 2 * V + V + j) * kThreads + threadIdx.x], g);
      Vec2<E>::unpack(gv[j], gn);
#pragma unroll
      for (int i = 0; i < N2; ++i) {
        x[i] = f2_mul(f2_add(x[i], nmu), r2);
        hh[i] = f2_mul(g[i], gn[i]);
      }
    };
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int k = from + ((j * W + w) * L + lane) * N;
      if (k < d) {
        F2 g[N2];
        constexpr int kKeep = kAgain ? 0 : 1;
        form(j, xh[kKeep * j], h[kKeep * j], g);
#pragma unroll
        for (int i = 0; i < N2; ++i) {
          a2 = f2_add(a2, h[kKeep * j][i]);
          b2 = f2_fma(h[kKeep * j][i], xh[kKeep * j][i], b2);
          dg[j][i] = f2_fma(g[i], xh[kKeep * j][i], dg[j][i]);
          db[j][i] = f2_add(db[j][i], g[i]);
        }
      }
    }
    float a = lane_sum<L>(f2_sum(a2)), b = lane_sum<L>(f2_sum(b2));
    if constexpr (C > 1) {
      // as below, with the other CTA's sums: every warp writes its own to both
      if (lane == 0) {
        sh[it][rank * W + w] = make_float2(a, b);
        store_remote(map_to_rank(smem_u32(&sh[it][rank * W + w]), rank ^ 1), a, b);
      }
      cluster_sync();
      a = b = 0.f;
#pragma unroll
      for (int i = 0; i < C * W; ++i) {
        const float2 v = sh[it][i];
        a += v.x;
        b += v.y;
      }
    } else if constexpr (W > 1) {
      // One barrier a row: the next row's words are the other half, and a warp comes back
      // to this one only past that row's barrier, when all have read it.
      if (lane == 0) sh[it][warp] = make_float2(a, b);
      group_sync(1 + group, 32 * W);
      a = b = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float2 v = sh[it][group * W + i];
        a += v.x;
        b += v.y;
      }
    }
    const F2 na = f2(-a * inv_d), nb = f2(-b * inv_d);
    E* dx = static_cast<E*>(p.dx) + t * p.d;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int k = from + ((j * W + w) * L + lane) * N;
      if (k < d) {
        constexpr int kKeep = kAgain ? 0 : 1;
        if constexpr (kAgain) {
          F2 g[N2];
          form(j, xh[0], h[0], g);
        }
#pragma unroll
        for (int i = 0; i < N2; ++i)
          h[kKeep * j][i] = f2_mul(f2_fma(xh[kKeep * j][i], nb, f2_add(h[kKeep * j][i], na)), r2);
        st16(dx + k, Vec2<E>::pack(h[kKeep * j]));
      }
    }
    slot = slot + 1 == S ? 0 : slot + 1;
  }
  copy_wait<0>();
  if constexpr (C > 1) cluster_sync();  // the other CTA's last words have arrived here
  chain_trigger();  // the second kernel's launch, under the last rows
  if (!p.part) return;
  if constexpr (kRows > 1) {  // the warp's rows into its first lanes
    static_assert(V == 1, "one vector a lane");
#pragma unroll
    for (int i = 0; i < N2; ++i)
#pragma unroll
      for (int o = L; o < 32; o <<= 1) {
        dg[0][i] = f2_add(dg[0][i], __shfl_xor_sync(0xffffffffu, dg[0][i], o));
        db[0][i] = f2_add(db[0][i], __shfl_xor_sync(0xffffffffu, db[0][i], o));
      }
  }

  // ---- the block's sums: its groups' one after the other
  float* out = p.part + 2ll * p.d * block;
  float* sums = reinterpret_cast<float*>(ring);
  __syncthreads();
  for (int q = 0; q < kGroups; ++q) {
    if (group == q && part == 0) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int k = from + ((j * W + w) * L + lane) * N;
        if (k < to) {
          float* s = q + 1 < kGroups ? sums : out;  // the last group writes the block's share
#pragma unroll
          for (int i = 0; i < N; i += 4) {
            float4 g, b;
            f2_split(dg[j][i / 2], g.x, g.y);
            f2_split(dg[j][i / 2 + 1], g.z, g.w);
            f2_split(db[j][i / 2], b.x, b.y);
            f2_split(db[j][i / 2 + 1], b.z, b.w);
            if (q > 0) {
              const float4 pg = *reinterpret_cast<const float4*>(sums + k + i);
              const float4 pb = *reinterpret_cast<const float4*>(sums + p.d + k + i);
              g = make_float4(g.x + pg.x, g.y + pg.y, g.z + pg.z, g.w + pg.w);
              b = make_float4(b.x + pb.x, b.y + pb.y, b.z + pb.z, b.w + pb.w);
            }
            *reinterpret_cast<float4*>(s + k + i) = g;
            *reinterpret_cast<float4*>(s + p.d + k + i) = b;
          }
        }
      }
    }
    __syncthreads();
  }
}

// Blocks' shares [splits][2][d] -> dgain, dbias.  A block owns 32 vectors of four columns;
// each of its 16 warps adds every 16th share, ten at a time (152 shares: one
// memory latency), then the first adds the warps'.
constexpr int kColWarps = 16, kColBatch = 10;

__global__ void __launch_bounds__(32 * kColWarps) norm_cols_sum_kernel(const NormParams p) {
  __shared__ float4 sh[kColWarps][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int c = (blockIdx.x * 32 + lane) * 4;
  chain_wait();
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < 2 * p.d) {
    const float* part = p.part + c;
    for (int s0 = warp; s0 < p.splits; s0 += kColWarps * kColBatch) {
      float4 v[kColBatch];
#pragma unroll
      for (int i = 0; i < kColBatch; ++i) {
        const int s = s0 + i * kColWarps;
        v[i] = s < p.splits ? *reinterpret_cast<const float4*>(part + 2ll * p.d * s) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int i = 0; i < kColBatch; ++i) a = make_float4(a.x + v[i].x, a.y + v[i].y, a.z + v[i].z, a.w + v[i].w);
    }
  }
  sh[warp][lane] = a;
  __syncthreads();
  if (warp > 0 || c >= 2 * p.d) return;
  for (int i = 1; i < kColWarps; ++i) {
    const float4 b = sh[i][lane];
    a = make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
  }
  float* out = c < p.d ? p.dgain : p.dbias;  // d is a multiple of 4: a vector lies in one of them
  if (!out) return;
  const int k = c < p.d ? c : c - p.d;
  out[k] = a.x;
  out[k + 1] = a.y;
  out[k + 2] = a.z;
  out[k + 3] = a.w;
}

// ------------------------------------------------------------------ wide rows
// A lane adds d / 32 values, a thread of the column sums T / splits rows, with no bound on either but
// 32 bits: a few at a time in fp32, and those in two words (one fp32 chain of 2^17 equal squares was
// off by 6e-4).
constexpr int kWarps = 4;

// A row's sum from the lanes', in every lane.
__device__ __forceinline__ float wide_sum(Pair v) { return __shfl_sync(0xffffffffu, pair_float(warp_sum_pair(v)), 0); }

template <typename E>
__global__ void __launch_bounds__(32 * kWarps) norm_fwd_wide_kernel(const NormParams p) {
  constexpr int N = Vec<E>::N;
  const long long t = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= p.T) return;
  const E* x = static_cast<const E*>(p.x) + t * p.d;
  const E* gain = static_cast<const E*>(p.gain);
  const E* bias = static_cast<const E*>(p.bias);
  E* y = static_cast<E*>(p.y) + t * p.d;
  const float inv_d = 1.0f / static_cast<float>(p.d);
  float f[N];
  Pair s = {0.f, 0.f}, q = {0.f, 0.f};
  for (int k = lane * N; k < p.d; k += 32 * N) {
    Vec<E>::unpack(ld16(x + k), f);
    float some = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) some += f[i];
    pair_add(s, some, 0.f);
  }
  const float mu = wide_sum(s) * inv_d;
  for (int k = lane * N; k < p.d; k += 32 * N) {
    Vec<E>::unpack(ld16(x + k), f);
    float some = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) some = fmaf(f[i] - mu, f[i] - mu, some);
    pair_add(q, some, 0.f);
  }
  const float r = 1.0f / sqrtf(wide_sum(q) * inv_d + p.eps);
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
__global__ void __launch_bounds__(32 * kWarps) norm_bwd_wide_kernel(const NormParams p) {
  constexpr int N = Vec<E>::N;
  const long long t = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= p.T) return;
  const E* x = static_cast<const E*>(p.x) + t * p.d;
  const E* dy = static_cast<const E*>(p.dy) + t * p.d;
  const E* gain = static_cast<const E*>(p.gain);
  E* dx = static_cast<E*>(p.dx) + t * p.d;
  const float inv_d = 1.0f / static_cast<float>(p.d), mu = p.mean[t], r = p.rstd[t];
  float f[N], h[N], g[N];
  Pair sa = {0.f, 0.f}, sb = {0.f, 0.f};
  for (int k = lane * N; k < p.d; k += 32 * N) {
    Vec<E>::unpack(ld16(x + k), f);
    Vec<E>::unpack(ld16(dy + k), h);
    if (gain) Vec<E>::unpack(ld16(gain + k), g);
    float some_a = 0.f, some_b = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float hg = gain ? h[i] * g[i] : h[i];
      some_a += hg;
      some_b = fmaf(hg, (f[i] - mu) * r, some_b);
    }
    pair_add(sa, some_a, 0.f);
    pair_add(sb, some_b, 0.f);
  }
  const float a = wide_sum(sa) * inv_d, b = wide_sum(sb) * inv_d;
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

// Column sums: a thread owns a column (x), a block every splits-th row (y), kColRows of them at a time.
constexpr int kColThreads = 128, kColRows = 8;

template <typename E>
__global__ void __launch_bounds__(kColThreads) norm_cols_wide_kernel(const NormParams p) {
  const int c = blockIdx.x * kColThreads + threadIdx.x;
  if (c >= p.d) return;
  const E* x = static_cast<const E*>(p.x);
  const E* dy = static_cast<const E*>(p.dy);
  Pair dg = {0.f, 0.f}, db = {0.f, 0.f};
  long long t = blockIdx.y;
  const long long step = p.splits;
  for (; t + (kColRows - 1) * step < p.T; t += kColRows * step) {
    float g[kColRows], v[kColRows], mu[kColRows], r[kColRows];
#pragma unroll
    for (int i = 0; i < kColRows; ++i) {  // every load before the first is used
      const long long row = t + i * step;
      g[i] = static_cast<float>(dy[row * p.d + c]);
      v[i] = static_cast<float>(x[row * p.d + c]);
      mu[i] = p.mean[row];
      r[i] = p.rstd[row];
    }
    float some_g = 0.f, some_b = 0.f;
#pragma unroll
    for (int i = 0; i < kColRows; ++i) {
      some_g = fmaf(g[i], (v[i] - mu[i]) * r[i], some_g);
      some_b += g[i];
    }
    pair_add(dg, some_g, 0.f);
    pair_add(db, some_b, 0.f);
  }
  for (; t < p.T; t += step) {
    const float g = static_cast<float>(dy[t * p.d + c]);
    pair_add(dg, g * ((static_cast<float>(x[t * p.d + c]) - p.mean[t]) * p.rstd[t]), 0.f);
    pair_add(db, g, 0.f);
  }
  float* out = p.part + 2ll * p.d * blockIdx.y + c;
  out[0] = pair_float(dg);
  out[p.d] = pair_float(db);
}

unsigned blocks_of(long long n, int per) { return static_cast<unsigned>((n + per - 1) / per); }

template <typename E, int V, int W, int L = 32>
cudaError_t fwd(const NormParams& p, cudaStream_t s) {
  norm_fwd_kernel<E, V, W, L><<<blocks_of(p.T, kFwdGroups<W> * (32 / L)), 32 * W * kFwdGroups<W>, 0, s>>>(p);
  return cudaGetLastError();
}

template <typename E>
cudaError_t fwd_any(const NormParams& p, cudaStream_t s) {
  if (p.d <= 8 * Vec<E>::N) return fwd<E, 1, 1, 8>(p, s);
  if (p.d <= 16 * Vec<E>::N) return fwd<E, 1, 1, 16>(p, s);
  // As few vectors a lane as the row needs, in as few warps as hold them: registers bound
  // the rows in flight, and a row's second warp costs two barriers.  16384 bf16 rows of 1032
  // values: 5 vectors in 1 warp 15 us, 8 in 1 18, 2 in 4 20, 3 in 2 26; of 2056: 3 in 4 28, 4
  // in 4 31; of 4104: 5 in 4 45, 4 in 8 67; of 8200: 5 in 8 105, 4 in 16 155; of 12288: 6 in
  // 8 126, 8 in 8 164.  32768 of 2048: 8 in 1 and 2 in 4 45, 4 in 2 60.
  const int v = (p.d + 32 * Vec<E>::N - 1) / (32 * Vec<E>::N);  // vectors a lane of one warp
  if (v <= 1) return fwd<E, 1, 1>(p, s);
  if (v <= 2) return fwd<E, 2, 1>(p, s);
  if (v <= 3) return fwd<E, 3, 1>(p, s);
  if (v <= 4) return fwd<E, 4, 1>(p, s);
  if (v <= 5) return fwd<E, 5, 1>(p, s);
  if (v <= 6) return fwd<E, 6, 1>(p, s);
  if (v <= 8) return fwd<E, 2, 4>(p, s);
  if (v <= 12) return fwd<E, 3, 4>(p, s);
  if (v <= 16) return fwd<E, 4, 4>(p, s);
  if (v <= 20) return fwd<E, 5, 4>(p, s);
  if (v <= 24) return fwd<E, 6, 4>(p, s);
  if (v <= 32) return fwd<E, 8, 4>(p, s);
  if (v <= 40) return fwd<E, 5, 8>(p, s);
  if (v <= 48) return fwd<E, 6, 8>(p, s);
  if (v <= 64) return fwd<E, 8, 8>(p, s);
  if (v <= 96) return fwd<E, 6, 16>(p, s);
  if (v <= 128) return fwd<E, 8, 16>(p, s);
  norm_fwd_wide_kernel<E><<<blocks_of(p.T, kWarps), 32 * kWarps, 0, s>>>(p);
  return cudaGetLastError();
}

// Rows of a lane's vectors in the ring: as many as 160 KB hold, at most 8.
template <int V>
constexpr int kRows = V >= 4 ? 3 : V == 3 ? 4 : V == 2 ? 5 : 8;
template <int V>
constexpr size_t kRingBytes = sizeof(uint4) * 2 * V * 32 * kBwdWarps * kRows<V>;

template <typename E, int V, int W, int L = 32, int C = 1>
cudaError_t bwd(const NormParams& p, cudaStream_t s) {
  static_assert(sizeof(float) * 2 * V * W * 32 * Vec<E>::N <= kRingBytes<V>, "the sums fit in the ring's memory");
  if constexpr (C == 1) {
    norm_bwd_kernel<E, V, W, kRows<V>, L, 1><<<p.splits, 32 * kBwdWarps, kRingBytes<V>, s>>>(p);
    return cudaGetLastError();
  } else {
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = C;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(C * p.splits);
    cfg.blockDim = dim3(32 * kBwdWarps);
    cfg.dynamicSmemBytes = kRingBytes<V>;
    cfg.stream = s;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, norm_bwd_kernel<E, V, W, kRows<V>, L, C>, p);
    if (e != cudaSuccess) cudaGetLastError();
    return e;
  }
}

// The cached backward's rows: at most 16 warps of 4 vectors a lane in each of two CTAs.
int lane_vectors(int d, bool fp32) { return (d + 32 * (fp32 ? 4 : 8) - 1) / (32 * (fp32 ? 4 : 8)); }
bool bwd_cached(int d, bool fp32) { return lane_vectors(d, fp32) <= 2 * 64; }

template <typename E>
cudaError_t bwd_any(const NormParams& p, cudaStream_t s) {
  if (p.d <= 8 * Vec<E>::N) return bwd<E, 1, 1, 8>(p, s);
  if (p.d <= 16 * Vec<E>::N) return bwd<E, 1, 1, 16>(p, s);
  // 2 or 3 vectors a lane: 16384 bf16 rows of 2056 values 54 -> 47 us against 2 in twice the
  // warps, of 6000 118 -> 98, of 12288 282 (4 in 16 warps) -> 186; but one warp with 3 takes
  // 26 us for 768, two with 2 take 22.
  const int v = lane_vectors(p.d, Vec<E>::N == 4);
  if (v <= 1) return bwd<E, 1, 1>(p, s);
  if (v <= 2) return bwd<E, 2, 1>(p, s);
  if (v <= 4) return bwd<E, 2, 2>(p, s);
  if (v <= 6) return bwd<E, 3, 2>(p, s);
  if (v <= 8) return bwd<E, 2, 4>(p, s);
  if (v <= 12) return bwd<E, 3, 4>(p, s);
  if (v <= 16) return bwd<E, 2, 8>(p, s);
  if (v <= 24) return bwd<E, 3, 8>(p, s);
  if (v <= 32) return bwd<E, 2, 16>(p, s);
  if (v <= 48) return bwd<E, 3, 16>(p, s);
  // bf16 rows of up to 16384 values split over two CTAs too: 16384 x 16384 took 426 us, a
  // row's exchange through the cluster being 0.6 of the 2 us that the row takes
  if (v <= 64) return bwd<E, 4, 16>(p, s);
  if (v <= 96) return bwd<E, 3, 16, 32, 2>(p, s);
  return bwd<E, 4, 16, 32, 2>(p, s);
}

}  // namespace

// Shares of the column sums: the cached backward's blocks (clusters, where rows are split),
// as many as its groups of warps need for one row each and at most what the SMs hold.
int norm_splits(long long T, int d, bool fp32, int sms) {
  if (bwd_cached(d, fp32)) {
    const int n = fp32 ? 4 : 8, v = lane_vectors(d, fp32);
    const int rows = d <= 8 * n ? 4 * kBwdWarps : d <= 16 * n ? 2 * kBwdWarps  // of a block at a time
                     : kBwdWarps / (v <= 2 ? 1 : v <= 6 ? 2 : v <= 12 ? 4 : v <= 24 ? 8 : 16);
    const long long blocks = (T + rows - 1) / rows;
    const int most = v > 64 ? (sms + 1) / 2 : sms;
    return blocks < 1 ? 1 : blocks < most ? static_cast<int>(blocks) : most;
  }
  const long long cols = (d + kColThreads - 1) / kColThreads;
  long long s = (8ll * sms + cols - 1) / cols;
  if (s > (T + 15) / 16) s = (T + 15) / 16;
  return s < 1 ? 1 : static_cast<int>(s);
}

cudaError_t launch_norm_fwd(const NormParams& p, bool fp32, cudaStream_t s) {
  if (p.T <= 0) return cudaSuccess;
  return fp32 ? fwd_any<float>(p, s) : fwd_any<__nv_bfloat16>(p, s);
}

cudaError_t launch_norm_bwd(const NormParams& p, bool fp32, cudaStream_t s) {
  if (p.T <= 0) return cudaSuccess;
  const bool sums = p.dgain || p.dbias;
  cudaError_t e;
  if (bwd_cached(p.d, fp32)) {
    e = fp32 ? bwd_any<float>(p, s) : bwd_any<__nv_bfloat16>(p, s);
    if (e != cudaSuccess || !sums) return e;
  } else if (sums) {  // before dx, which may take dy's place
    const dim3 cols(blocks_of(p.d, kColThreads), p.splits);
    if (fp32)
      norm_cols_wide_kernel<float><<<cols, kColThreads, 0, s>>>(p);
    else
      norm_cols_wide_kernel<__nv_bfloat16><<<cols, kColThreads, 0, s>>>(p);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
  }
  if (sums && (e = launch_chained(norm_cols_sum_kernel, dim3(blocks_of(2 * p.d, 128)), dim3(32 * kColWarps), 0, s, p)) != cudaSuccess)
    return e;
  if (bwd_cached(p.d, fp32)) return cudaSuccess;
  const unsigned grid = blocks_of(p.T, kWarps);
  if (fp32)
    norm_bwd_wide_kernel<float><<<grid, 32 * kWarps, 0, s>>>(p);
  else
    norm_bwd_wide_kernel<__nv_bfloat16><<<grid, 32 * kWarps, 0, s>>>(p);
  return cudaGetLastError();
}

// Dynamic shared memory beyond 48 KB.
cudaError_t setup_norm_kernels() {
  cudaError_t e;
#define MLS_SET(K, BYTES)                                                                     \
  e = cudaFuncSetAttribute(K, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(BYTES)); \
  if (e != cudaSuccess) return e;
#define MLS_SET_RING(E, V, W, L, C) MLS_SET((norm_bwd_kernel<E, V, W, kRows<V>, L, C>), kRingBytes<V>)
#define MLS_SET_BOTH(V, W, L, C) MLS_SET_RING(float, V, W, L, C) MLS_SET_RING(__nv_bfloat16, V, W, L, C)
  MLS_SET_BOTH(1, 1, 8, 1)
  MLS_SET_BOTH(1, 1, 16, 1)
  MLS_SET_BOTH(1, 1, 32, 1)
  MLS_SET_BOTH(2, 1, 32, 1)
  MLS_SET_BOTH(2, 2, 32, 1)
  MLS_SET_BOTH(3, 2, 32, 1)
  MLS_SET_BOTH(2, 4, 32, 1)
  MLS_SET_BOTH(3, 4, 32, 1)
  MLS_SET_BOTH(2, 8, 32, 1)
  MLS_SET_BOTH(3, 8, 32, 1)
  MLS_SET_BOTH(2, 16, 32, 1)
  MLS_SET_BOTH(3, 16, 32, 1)
  MLS_SET_BOTH(4, 16, 32, 1)
  MLS_SET_BOTH(3, 16, 32, 2)
  MLS_SET_BOTH(4, 16, 32, 2)
#undef MLS_SET_BOTH
#undef MLS_SET_RING
#undef MLS_SET
  return cudaSuccess;
}

}  // namespace mls
