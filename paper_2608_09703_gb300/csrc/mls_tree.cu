// Attention of new tokens (the nodes of a drafted tree, a chain, or one token) over a paged
// key/value cache.  For node t of an entry, query head h and its key/value head:
//   out = sum_j softmax_j(scale q . k_j) v_j,   lse = log sum_j exp(scale q . k_j)
// over the entry's cached tokens and the nodes on the path from t to its root, t included.
#include <climits>
#include <cmath>

#include "mls_device.cuh"
#include "mls_kernels.h"
#include "mls_tree.cuh"
#include "mls_vec.cuh"

namespace mls {
namespace {

// ------------------------------------------------------------------ one warp a node
// A warp takes one node and up to kHeads query heads of one key/value head, a piece of the keys, 32
// of them at a time: each lane has a key, the products with the queries of the heads come from
// shared memory; then each lane has four columns of the values.  All heads of a node see the same keys,
// so what the mask leaves out is not even read.
constexpr int kHeads = 4, kWarps = 4;

template <typename E>
__device__ __forceinline__ void load4(const E* p, float (&f)[4]);
template <>
__device__ __forceinline__ void load4<float>(const float* p, float (&f)[4]) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w;
}
template <>
__device__ __forceinline__ void load4<__nv_bfloat16>(const __nv_bfloat16* p, float (&f)[4]) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  f[0] = __uint_as_float(v.x << 16), f[1] = __uint_as_float(v.x & 0xffff0000u);
  f[2] = __uint_as_float(v.y << 16), f[3] = __uint_as_float(v.y & 0xffff0000u);
}
__device__ __forceinline__ void store4(float* p, const float (&f)[4]) {
  *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float (&f)[4]) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

template <typename E>
__global__ void __launch_bounds__(32 * kWarps) node_kernel(TreeParams p) {
  __shared__ float qs[kWarps][kHeads][128];
  __shared__ short up[kWarps][kTreeMaxNodes];
  __shared__ unsigned see[kWarps][kTreeMaxNodes / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int chunks = (p.group + kHeads - 1) / kHeads;
  const long long per_node = static_cast<long long>(p.c.heads) * chunks * p.splits;
  const long long task = static_cast<long long>(blockIdx.x) * kWarps + warp;
  if (task >= p.N * per_node) return;
  const long long t = task / per_node;
  int rest = static_cast<int>(task - t * per_node);
  const int split = rest % p.splits;
  rest /= p.splits;
  const int chunk = rest % chunks, kvh = rest / chunks;
  const int h0 = kvh * p.group + chunk * kHeads, nh = min(kHeads, p.group - chunk * kHeads);
  int mine = -1;
  for (int i0 = 0; i0 < p.n && mine < 0; i0 += 32) {
    const int i = i0 + lane;
    const bool here = i < p.n && p.start[i] <= t && t < p.start[i + 1];
    const unsigned b = __ballot_sync(0xffffffffu, here);
    if (b) mine = i0 + __ffs(b) - 1;
  }
  if (mine < 0) return;  // behind the last entry: left as it was
  const Entry e = tree_entry(p, mine, p.status);
  const int node = static_cast<int>(t - e.first);
  bool used = e.row >= 0 && e.nodes > 0;
  if (used && p.parents) {
    for (int j = lane; j < e.nodes; j += 32) {
      const int u = p.parents[e.first + j];
      const bool odd = u < -2 || u >= j;
      if (odd) atomicOr(p.status, kStatusBadSeq);
      up[warp][j] = static_cast<short>(odd ? -2 : u);
    }
    if (lane < kTreeMaxNodes / 32) see[warp][lane] = 0u;
    __syncwarp();
    if (lane == 0)
      for (int j = node; j >= 0 && up[warp][j] >= -1; j = up[warp][j]) see[warp][j >> 5] |= 1u << (j & 31);
    used = up[warp][node] >= -1;
    __syncwarp();
  }
  for (int x = lane; x < nh * p.dim; x += 32) {
    const int h = x / p.dim, d = x - h * p.dim;
    const float f = static_cast<float>(static_cast<const E*>(p.q)[t * p.q_ld + static_cast<long long>(h0 + h) * p.dim + d]);
    qs[warp][h][d] = p.negate ? -f : f;
  }
  __syncwarp();
  float m[kHeads], l[kHeads], o[kHeads][4];
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    m[h] = -INFINITY;
    l[h] = 0.f;
    o[h][0] = o[h][1] = o[h][2] = o[h][3] = 0.f;
  }
  const int total = used ? e.len + node + 1 : 0;
  const int each = (total + 32 * p.splits - 1) / (32 * p.splits) * 32;
  const int k0 = static_cast<int>(min(static_cast<long long>(split) * each, static_cast<long long>(total)));
  const int k1 = static_cast<int>(min(static_cast<long long>(k0) + each, static_cast<long long>(total)));
  const int mask = (1 << p.c.page_shift) - 1;
  const E* const K = reinterpret_cast<const E*>(p.c.k);
  const E* const V = reinterpret_cast<const E*>(p.c.v);
  const int width = 16 / static_cast<int>(sizeof(E));  // values of a piece
  for (int b = k0; b < k1; b += 32) {
    const int pos = b + lane;
    bool seen = pos < k1;
    if (seen && pos >= e.len && p.parents) seen = see[warp][(pos - e.len) >> 5] >> ((pos - e.len) & 31) & 1u;
    long long at = -1;
    if (seen) {
      const int page = p.c.table[static_cast<long long>(e.row) * p.c.max_pages + (pos >> p.c.page_shift)];
      if (page >= 0 && page < p.c.pages) at = cache_at(p.c, p.layer, page, kvh, pos & mask) * width;
      else atomicOr(p.status, kStatusBadSeq);  // its keys and values count as 0
    }
    float s[kHeads] = {0.f, 0.f, 0.f, 0.f};
    if (at >= 0)
      for (int d = 0; d < p.dim; d += 4) {
        float f[4];
        load4(K + at + d, f);
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
          const float4 q = *reinterpret_cast<const float4*>(&qs[warp][h][d]);
          s[h] = fmaf(f[3], q.w, fmaf(f[2], q.z, fmaf(f[1], q.y, fmaf(f[0], q.x, s[h]))));
        }
      }
    float w[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      const float z = seen ? s[h] : -INFINITY;
      float top = z;
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      const float now = fmaxf(m[h], top);
      const float base = now == -INFINITY ? 0.f : now * p.scale;
      const float c = exp2f(fmaf(m[h], p.scale, -base));
      w[h] = seen ? exp2f(fmaf(z, p.scale, -base)) : 0.f;
      l[h] = fmaf(l[h], m[h] == -INFINITY ? 0.f : c, warp_sum(w[h]));
#pragma unroll
      for (int j = 0; j < 4; ++j) o[h][j] *= m[h] == -INFINITY ? 0.f : c;
      m[h] = now;
    }
    unsigned live = __ballot_sync(0xffffffffu, at >= 0);
    while (live) {
      const int k = __ffs(live) - 1;
      live &= live - 1u;
      const long long va = __shfl_sync(0xffffffffu, at, k);
      float f[4] = {0.f, 0.f, 0.f, 0.f};
      if (lane * 4 < p.dim) load4(V + va + lane * 4, f);
#pragma unroll
      for (int h = 0; h < kHeads; ++h) {
        const float wk = __shfl_sync(0xffffffffu, w[h], k);
#pragma unroll
        for (int j = 0; j < 4; ++j) o[h][j] = fmaf(wk, f[j], o[h][j]);
      }
    }
  }
  for (int h = 0; h < nh; ++h) {
    const long long row = t * p.q_heads + h0 + h;
    if (p.splits > 1) {
      float* const part = p.part + (row * p.splits + split) * (p.dim + 4);
      if (lane * 4 < p.dim) store4(part + 4 + lane * 4, o[h]);
      if (lane == 0) part[0] = m[h], part[1] = l[h];
      continue;
    }
    const float inv = l[h] == 0.f ? 0.f : 1.f / l[h];
#pragma unroll
    for (int j = 0; j < 4; ++j) o[h][j] *= inv;
    if (lane * 4 < p.dim) store4(static_cast<E*>(p.out) + row * p.dim + lane * 4, o[h]);
    if (lane == 0) p.lse[row] = l[h] == 0.f ? -INFINITY : fmaf(m[h], p.scale, log2f(l[h])) * kLn2;
  }
}

// Joins the pieces of a node's keys, in order.  A warp a node and head.
template <typename E>
__global__ void __launch_bounds__(32 * kWarps) join_kernel(TreeParams p) {
  chain_wait();
  const int lane = threadIdx.x & 31;
  const long long row = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  if (row >= p.N * p.q_heads || row / p.q_heads >= p.start[p.n] || row / p.q_heads < p.start[0]) return;
  const int stride = p.dim + 4;
  const float* const part = p.part + row * p.splits * stride;
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = lane; s < p.splits; s += 32) m = fmaxf(m, part[s * stride]);
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
  const float base = m == -INFINITY ? 0.f : m * p.scale;
  for (int s = 0; s < p.splits; ++s) {
    const float* const x = part + s * stride;
    if (x[1] == 0.f) continue;  // nothing seen
    const float c = x[0] == -INFINITY ? 1.f : exp2f(fmaf(x[0], p.scale, -base));  // a sum without a maximum is NaN
    l = fmaf(x[1], c, l);
    if (lane * 4 < p.dim) {
      float f[4];
      load4(x + 4 + lane * 4, f);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = fmaf(f[j], c, o[j]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] *= inv;
  if (lane * 4 < p.dim) store4(static_cast<E*>(p.out) + row * p.dim + lane * 4, o);
  if (lane == 0) p.lse[row] = l == 0.f ? -INFINITY : fmaf(m, p.scale, log2f(l)) * kLn2;
}

template <typename E>
cudaError_t run_nodes(const TreeParams& p, cudaStream_t s) {
  const long long tasks = p.N * p.c.heads * ((p.group + kHeads - 1) / kHeads) * p.splits;
  node_kernel<E><<<static_cast<unsigned>((tasks + kWarps - 1) / kWarps), 32 * kWarps, 0, s>>>(p);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || p.splits == 1) return e;
  return launch_chained(join_kernel<E>, dim3(static_cast<unsigned>((p.N * p.q_heads + kWarps - 1) / kWarps)),
                        dim3(32 * kWarps), 0, s, p);
}

}  // namespace

// Pieces of the keys: as many warps as the card holds sixteen an SM of, where the nodes are few.
int tree_fp32_splits(long long N, int q_heads, int sms) {
  const long long rows = N * ((q_heads + kHeads - 1) / kHeads);
  const long long want = rows > 0 ? (16LL * sms) / rows : 1;
  return static_cast<int>(want < 1 ? 1 : want > 64 ? 64 : want);
}

cudaError_t launch_tree_fp32(const TreeParams& p, cudaStream_t s) { return run_nodes<float>(p, s); }

}  // namespace mls
