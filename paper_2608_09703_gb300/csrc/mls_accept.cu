// Acceptance of a drafted tree's tokens against the target's probabilities, from given random
// numbers.  A walk begins at node 0 of a sequence.  At node i with target row p and draft row q its
// children are tried in order; child d with token x is accepted if u_d q(x) < r(x), where r = p at
// first and r <- max(0, r - q) / sum after each refusal (not where that is 0 everywhere).  Where none
// is accepted, the next token is drawn from r by inverse CDF.
//
// The residuals need no row of their own.  With r = w / Z, w_0 = p and Z_0 = 1,
//   w_{j+1} = max(0, w_j - Z_j q) = max(0, p - c_{j+1} q),   c_{j+1} = c_j + Z_j,  Z_j = sum w_j,
// since q >= 0.  (Siblings drawn without repetition: q_j = s_j q without the tokens refused so far, s_j
// = 1 / sum of what is left of q; then c_{j+1} = c_j + s_j Z_j, and a refused token keeps the c of its
// refusal.  A draft without probabilities: q is 1 at the token; w is p without the tokens refused.)
// So a refusal costs one pass over two rows and no store, and acceptance needs one value of each
// row per node, all of which are fetched before the walk begins.
//
// Which token an inverse CDF finds depends on where its sums' edges lie, so the sums are taken in two
// fp32 words, p - c q too, and decisions are made in 64 bits: a handful per node.  (64-bit sums of a
// row of 50304 would take an SM's two units 12 us.)
// A sequence has a cluster of CTAs, each with a part of the vocabulary, whose warps' sums meet in
// shared memory; all walk alike.
#include <climits>
#include <cstddef>

#include "mls_device.cuh"
#include "mls_kernels.h"
#include "mls_vec.cuh"

namespace mls {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kSpan = 128;  // values that a warp reads at a time

// What the walk asks of all threads: sums over the row of node `row`, and whether a token is then
// drawn from them.
struct Pass {
  int row, refused;
  float c_hi, c_lo;              // c of the tokens that were not refused
  bool read, with_draft, draw;   // sums are needed; p - c q, not p; they are the last
};
struct Walk {
  int parent[kTreeMaxNodes], token[kTreeMaxNodes];
  float u[kTreeMaxNodes], p[kTreeMaxNodes], q[kTreeMaxNodes];  // p, q: of a node's token in its parent's rows
  int refused[kTreeMaxNodes];                                  // the tokens refused at the present node
  float c_hi[kTreeMaxNodes], c_lo[kTreeMaxNodes];              // and their c
  Pass pass;
  // Of every warp of the cluster: its sum of w, and of what is left of q.  Two of each: a CTA may begin the
  // next pass while another still reads the sums of this one.
  alignas(8) Pair sums[2][kMaxCluster * kWarps];               // written from other CTAs, two words at a time
  alignas(8) Pair mass[2][kMaxCluster * kWarps];
  Pair warp_sums[kWarps];
  double before, goal;           // of the part that holds the token drawn: the sum before it, u times the whole
  int part, found, last;
};

static_assert(offsetof(Walk, sums) % 8 == 0 && offsetof(Walk, mass) % 8 == 0, "stores of two words");

__device__ __forceinline__ Pair two(float v) { return {v, 0.f}; }
__device__ __forceinline__ void split(double v, float& hi, float& lo) {
  hi = static_cast<float>(v);
  lo = static_cast<float>(v - static_cast<double>(hi));
}
// p - c q in two words, nothing where that is not positive.
__device__ __forceinline__ Pair residual(float p, float q, float c_hi, float c_lo) {
  const float a = __fmul_rn(c_hi, q), b = fmaf(c_hi, q, -a) + c_lo * q;
  const float d = __fsub_rn(p, a), e = __fsub_rn(d, p);
  const float rest = __fadd_rn(__fsub_rn(p, __fsub_rn(d, e)), -__fadd_rn(a, e)) - b;
  const bool some = __fadd_rn(d, rest) > 0.f;
  return {some ? d : 0.f, some ? rest : 0.f};
}

// Whether token v was refused at this node (its place in the list, else -1).
__device__ __forceinline__ int refused_at(const Walk& s, int refused, int v) {
  for (int j = 0; j < refused; ++j)
    if (s.refused[j] == v) return j;
  return -1;
}
// w of token v, and what is left there of the draft's row.
template <bool kDraft>
__device__ __forceinline__ Pair value(const Walk& s, const Pass& a, float p, float& q, int v) {
  float hi = a.c_hi, lo = a.c_lo;
  const int j = a.refused ? refused_at(s, a.refused, v) : -1;
  if (j >= 0) {
    if (!kDraft) return two(0.f);
    hi = s.c_hi[j];
    lo = s.c_lo[j];
  }
  const Pair w = kDraft ? residual(p, q, hi, lo) : two(p);
  if (j >= 0) q = 0.f;
  return w;
}

// pair_add and residual of two values at a time.
struct Pair2 {
  float2 hi, lo;
};
__device__ __forceinline__ void pair2_add(Pair2& a, const float2& hi, const float2& lo) {
  const float2 s = add2(a.hi, hi), b = sub2(s, a.hi);
  a.lo = add2(a.lo, add2(add2(sub2(a.hi, sub2(s, b)), sub2(hi, b)), lo));
  a.hi = s;
}
__device__ __forceinline__ Pair2 residual2(const float2& p, const float2& q, float c_hi, float c_lo) {
  const float2 hi = make_float2(c_hi, c_hi);
  const float2 na = mul2(make_float2(-c_hi, -c_hi), q), b = fma2(make_float2(c_lo, c_lo), q, fma2(hi, q, na));
  const float2 d = add2(p, na), e = sub2(d, p);
  const float2 rest = sub2(sub2(sub2(p, sub2(d, e)), sub2(e, na)), b), all = add2(d, rest);
  const bool x = all.x > 0.f, y = all.y > 0.f;
  return {make_float2(x ? d.x : 0.f, y ? d.y : 0.f), make_float2(x ? rest.x : 0.f, y ? rest.y : 0.f)};
}

// The sums of a pass over this warp's part [v0, v1) of the row, to every CTA of the cluster.  Arithmetic bounds it
// (some 16 operations a value), so it is done on two values an instruction, and only stretches with a refused
// token look at which it is.
template <bool kDraft, bool kMass>
__device__ void row_pass(const AcceptParams& p, Walk& s, const Pass& a, long long row, long long v0, long long v1,
                         int buffer, int slot) {
  const int lane = threadIdx.x & 31;
  const float* const P = p.target + row * p.ld_target;
  const float* const Q = kDraft ? p.draft + row * p.ld_draft : nullptr;
  const float2 zero = make_float2(0.f, 0.f);
  Pair2 sum = {zero, zero}, mass = {zero, zero};
  constexpr int kDeep = 8;
  for (long long b0 = v0; b0 < v1; b0 += 32 * kDeep) {
    const long long b = b0 + lane;
    float x[kDeep], y[kDeep];
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
      const bool in = b + 32 * j < v1;
      x[j] = in ? P[b + 32 * j] : 0.f;
      y[j] = in && kDraft ? Q[b + 32 * j] : 0.f;
    }
    bool some = false;
    for (int j = 0; j < a.refused; ++j) some |= s.refused[j] >= b0 && s.refused[j] < b0 + 32 * kDeep;
#pragma unroll
    for (int j = 0; j < kDeep; j += 2) {
      Pair2 w = {make_float2(x[j], x[j + 1]), zero};
      if (some) {
        const Pair w0 = value<kDraft>(s, a, x[j], y[j], static_cast<int>(b + 32 * j));
        const Pair w1 = value<kDraft>(s, a, x[j + 1], y[j + 1], static_cast<int>(b + 32 * j + 32));
        w = {make_float2(w0.hi, w1.hi), make_float2(w0.lo, w1.lo)};
      } else if (kDraft) {
        w = residual2(w.hi, make_float2(y[j], y[j + 1]), a.c_hi, a.c_lo);
      }
      pair2_add(sum, w.hi, w.lo);
      if (kMass) pair2_add(mass, make_float2(y[j], y[j + 1]), zero);
    }
  }
  auto total = [](const Pair2& t) {
    Pair one = {t.hi.x, t.lo.x};
    pair_add(one, t.hi.y, t.lo.y);
    return warp_sum_pair(one);
  };
  const Pair one = total(sum), left = kMass ? total(mass) : two(0.f);
  if (lane == 0)
    for (int r = 0; r < p.cluster; ++r) {
      store_remote(map_to_rank(smem_u32(&s.sums[buffer][slot]), r), one.hi, one.lo);
      if (kMass) store_remote(map_to_rank(smem_u32(&s.mass[buffer][slot]), r), left.hi, left.lo);
    }
}

// Inclusive sums over the lanes.
__device__ __forceinline__ Pair warp_scan_pair(Pair a) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const float hi = __shfl_up_sync(0xffffffffu, a.hi, o), lo = __shfl_up_sync(0xffffffffu, a.lo, o);
    if (lane >= o) pair_add(a, hi, lo);
  }
  return a;
}
constexpr int kEach = kMaxCluster * kWarps / 32;  // warps' sums that a lane has
static_assert(kMaxCluster * kWarps % 32 == 0, "a lane's share");
// A lane's share of the warps' sums of a pass, and those up to it.
struct Sums {
  Pair mine, upto;
  __device__ __forceinline__ Sums(const Pair* x, int warps) : mine(two(0.f)) {
    const int at = (threadIdx.x & 31) * kEach;
    for (int j = 0; j < kEach; ++j)
      if (at + j < warps) pair_add(mine, x[at + j].hi, x[at + j].lo);
    upto = warp_scan_pair(mine);
  }
  __device__ __forceinline__ double total() const {
    return pair_value({__shfl_sync(0xffffffffu, upto.hi, 31), __shfl_sync(0xffffffffu, upto.lo, 31)});
  }
};

// Which warp's part holds the token that u draws from the sums.  Warp 0 calls it.
__device__ void choose_part(Walk& s, const Pair* sums, int warps, float u) {
  const int lane = threadIdx.x & 31;
  const Sums own(sums, warps);
  const double goal = static_cast<double>(u) * own.total(), end = pair_value(own.upto), mine = pair_value(own.mine);
  // The first lane whose sum passes the goal; of rounding, another's begin may be past it by a little.
  const unsigned past = __ballot_sync(0xffffffffu, end > goal && mine > 0.0);
  if (lane == 0) s.part = -1;
  __syncwarp();
  if (past && lane == __ffs(past) - 1) {
    double at = end - mine;
    int part = -1;
    for (int j = 0; j < kEach && lane * kEach + j < warps; ++j) {
      const double v = pair_value(sums[lane * kEach + j]);
      if (!(v > 0.0)) continue;
      part = lane * kEach + j;
      s.before = at;
      at += v;
      if (at > goal) break;
    }
    s.part = part;
    s.goal = goal;
  }
  __syncwarp();
}

// The token of part [v0, v1): the smallest v whose sum up to it, on top of s.before, is past s.goal.
template <bool kDraft>
__device__ void draw(const AcceptParams& p, Walk& s, const Pass& a, long long row, long long v0, long long v1, int* next) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float* const P = p.target + row * p.ld_target;
  const float* const Q = kDraft ? p.draft + row * p.ld_draft : nullptr;
  const long long each = (v1 - v0 + kThreads - 1) / kThreads;
  const long long a0 = min(v0 + tid * each, v1), a1 = min(a0 + each, v1);
  Pair sum = two(0.f);
  int first = -1, last = -1;
#pragma unroll 4
  for (long long v = a0; v < a1; ++v) {
    float q = kDraft ? Q[v] : 0.f;
    const Pair w = value<kDraft>(s, a, P[v], q, static_cast<int>(v));
    if (w.hi + w.lo > 0.f) {
      last = static_cast<int>(v);
      if (first < 0) first = last;
    }
    pair_add(sum, w.hi, w.lo);
  }
  if (tid == 0) s.found = INT_MAX, s.last = -1;
  const Pair upto = warp_scan_pair(sum);
  if (lane == 31) s.warp_sums[warp] = upto;
  __syncthreads();
  Pair base = two(0.f);
  for (int w = 0; w < warp; ++w) pair_add(base, s.warp_sums[w].hi, s.warp_sums[w].lo);
  if (last >= 0) atomicMax(&s.last, last);
  const double goal = s.goal, end = s.before + pair_value(base) + pair_value(upto), begin = end - pair_value(sum);
  if (end > goal && last >= 0) {
    if (begin > goal) {
      atomicMin(&s.found, first);
    } else {
      Pair cum = two(0.f);
      for (long long v = a0; v < a1; ++v) {
        float q = kDraft ? Q[v] : 0.f;
        const Pair w = value<kDraft>(s, a, P[v], q, static_cast<int>(v));
        if (!(w.hi + w.lo > 0.f)) continue;
        pair_add(cum, w.hi, w.lo);
        if (begin + pair_value(cum) > goal) {
          atomicMin(&s.found, static_cast<int>(v));
          break;
        }
      }
    }
  }
  __syncthreads();
  MLS_CHECK(p.status, s.found == INT_MAX ? s.last >= v0 && s.last < v1 : s.found >= v0 && s.found < v1);
  if (tid == 0) *next = s.found != INT_MAX ? s.found : s.last;  // the goal within rounding of the part's end
}

__global__ void __launch_bounds__(kThreads, 4) accept_kernel(AcceptParams p) {
  __shared__ Walk s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = p.cluster > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int b = blockIdx.x / p.cluster;
  const long long first = p.start[b], end = p.start[b + 1];
  const bool drafted = p.draft != nullptr, distinct = drafted && !p.replace;
  if (p.cluster > 1) cluster_arrive();  // a CTA's shared memory is written once it runs
  bool bad = first < 0 || end < first || end > p.N || end - first > kTreeMaxNodes || end - first > p.max_path;
  const int n = bad ? 0 : static_cast<int>(end - first);
  for (int j = tid; j < n; j += kThreads) {
    const int up = p.parents[first + j], x = p.tokens[first + j];
    const bool odd = up < -2 || up >= j || (j == 0 && up != -1);
    bad |= odd;
    s.parent[j] = odd ? -2 : up;
    s.token[j] = x;
    s.u[j] = p.u[2 * (first + j)];
    const bool in = !odd && up >= 0 && x >= 0 && x < p.V;
    s.p[j] = in ? p.target[(first + up) * p.ld_target + x] : 0.f;
    s.q[j] = in ? (drafted ? p.draft[(first + up) * p.ld_draft + x] : 1.f) : 0.f;  // outside: refused
  }
  int* const path = p.path + static_cast<long long>(b) * p.max_path;
  if (rank == 0)
    for (int j = tid; j < p.max_path; j += kThreads) path[j] = j == 0 && n > 0 ? 0 : -1;
  bad = __syncthreads_or(bad);
  if (rank == 0 && tid == 0) {
    if (bad) atomicOr(p.status, kStatusBadSeq);
    p.next[b] = -1;
    if (n == 0) p.n_path[b] = 0;
  }
  __syncwarp();
  if (p.cluster > 1) cluster_wait();
  if (n == 0) return;  // every CTA of the cluster
  // The part of the vocabulary of each of the cluster's warps, in order.
  const int warps = p.cluster * kWarps, slot = rank * kWarps + warp;
  const long long spans = (p.V + kSpan - 1) / kSpan, each = (spans + warps - 1) / warps * kSpan;
  const long long v0 = min(slot * each, p.V), v1 = min(v0 + each, p.V);

  // The walk, by warp 0 of every CTA alike: at node cur, whose children from `from` on are left.
  int cur = 0, from = 1, depth = 1, refused = 0, buffer = 1;
  double c = 0.0, c_old = 0.0, Z = 1.0, share = 1.0;
  bool pending = false, listed = false, fresh = false;  // a refusal's sums are due; they fit the present w
  while (true) {
    if (warp == 0) {
      if (pending) {
        const double sum = Sums(s.sums[buffer], warps).total();
        fresh = sum > 0.0;
        if (fresh) {
          Z = sum;
        } else {  // nothing left: the refusal leaves r as it was
          c = c_old;
          if (listed && !drafted) --refused;
          if (listed && drafted && lane == 0) split(c_old, s.c_hi[refused - 1], s.c_lo[refused - 1]);
        }
        if (distinct) {
          const double left = Sums(s.mass[buffer], warps).total();
          share = left > 0.0 ? 1.0 / left : 0.0;
        }
        pending = false;
        __syncwarp();
      }
      while (!pending) {
        int d = n;
        for (int j0 = from & ~31; j0 < n; j0 += 32) {
          const int j = j0 + lane;
          const unsigned hit = __ballot_sync(0xffffffffu, j >= from && j < n && s.parent[j] == cur);
          if (hit) {
            d = j0 + __ffs(hit) - 1;
            break;
          }
        }
        if (d == n) break;
        from = d + 1;
        const int x = s.token[d];
        const bool again = (distinct || !drafted) && refused_at(s, refused, x) >= 0;
        const double q = again && drafted ? 0.0 : share * s.q[d];
        double w = s.p[d];
        if (drafted) w = fma(-c, static_cast<double>(s.q[d]), w);
        else if (again) w = 0.0;
        if (q > 0.0 && static_cast<double>(s.u[d]) * q * Z < w) {
          cur = d;
          MLS_CHECK(p.status, depth < n && d < n);
          if (rank == 0 && lane == 0) path[depth] = d;
          ++depth;
          refused = 0;
          c = 0.0;
          Z = share = 1.0;
          fresh = false;
        } else if (drafted || (x >= 0 && x < p.V && !again)) {
          c_old = c;
          c += share * Z;
          listed = (distinct || !drafted) && x >= 0 && x < p.V && !again;
          MLS_CHECK(p.status, refused < kTreeMaxNodes);
          if (listed && lane == 0) {
            s.refused[refused] = x;
            split(c, s.c_hi[refused], s.c_lo[refused]);
          }
          refused += listed;
          pending = true;
        }
        __syncwarp();
      }
      if (lane == 0) {
        Pass a;
        a.row = cur;
        a.refused = refused;
        split(c, a.c_hi, a.c_lo);
        a.draw = !pending;
        a.read = !fresh || pending;
        a.with_draft = drafted && (pending || refused > 0 || c > 0.0);
        s.pass = a;
      }
    }
    __syncthreads();
    const Pass a = s.pass;
    const long long row = first + a.row;
    if (a.read) {
      buffer ^= 1;
      if (!a.with_draft) row_pass<false, false>(p, s, a, row, v0, v1, buffer, slot);
      else if (distinct) row_pass<true, true>(p, s, a, row, v0, v1, buffer, slot);
      else row_pass<true, false>(p, s, a, row, v0, v1, buffer, slot);
      __syncwarp();
      if (p.cluster > 1) cluster_sync();
      else __syncthreads();
    }
    if (!a.draw) continue;
    if (warp == 0) {
      choose_part(s, s.sums[buffer], warps, p.u[2 * row + 1]);
      if (rank == 0 && lane == 0) p.n_path[b] = depth;
    }
    __syncthreads();
    const int part = s.part;
    MLS_CHECK(p.status, part < warps);
    if (part < 0 || part / kWarps != rank) return;  // -1: a row without mass
    const long long b0 = min(part * each, p.V), b1 = min(b0 + each, p.V);
    if (a.with_draft) draw<true>(p, s, a, row, b0, b1, p.next + b);
    else draw<false>(p, s, a, row, b0, b1, p.next + b);
    return;
  }
}

}  // namespace

cudaError_t launch_accept(const AcceptParams& p, cudaStream_t s) {
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = p.cluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.n) * p.cluster);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, accept_kernel, p);
  if (e != cudaSuccess) cudaGetLastError();
  return e;
}

// Enough CTAs of a sequence that few sequences fill the card too, four an SM, but no fewer than 16 values a thread.
// (CTAs of 512 threads, one an SM: 102 chains at V = 50304 28.7 us, 64 trees at V = 128256 54 after the pass was packed;
// of 256, two an SM: 28.6 and 72; four: 22.5 and 50.)
int accept_cluster(int n, long long V, int sms) {
  int c = 1;
  while (c < kMaxCluster && static_cast<long long>(n) * 2 * c <= 4 * sms && V / (2 * c) >= 4096) c *= 2;
  return c;
}

}  // namespace mls
