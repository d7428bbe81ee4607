// Attention of new tokens (the nodes of a drafted tree, a chain, or one token) over a paged
// key/value cache.  For node t of an entry, query head h and its key/value head:
//   out = sum_j softmax_j(scale q . k_j) v_j,   lse = log sum_j exp(scale q . k_j)
// over the entry's cached tokens and the nodes on the path from t to its root, t included.
// Here: the kernel of an fp32 cache, and the one that joins pieces (a bf16 cache's: mls_tree_mma.cu).
//
// fp32: products of full precision are the vector units' work.  An item has 16 rows (4, where entries have no more:
// decoding) and tiles of 64 keys, of which each of eight warps has 8.  Half a warp has half of the rows, and a lane
// of it 8 columns, of the queries and of the product, in registers; a key's partial scores are added up by exchanges
// that leave each lane one row.  That asks shared memory for 8 of the 16 words a key and lane that it does for each of
// K and V (with rows over four groups of lanes and queries in shared memory 64 single tokens over 10000 took 766 us, now
// 528: 99% of the copy rate; 8 nodes of 16 heads over 30000 340 us, now 281).  Warps keep a maximum,
// sum and product of their own to the end of a segment.
#include <cmath>

#include "mls_device.cuh"
#include "mls_kernels.h"
#include "mls_tree.cuh"
#include "mls_vec.cuh"

namespace mls {
namespace {

constexpr int kWarps = 8, kKeys = 64, kThreads = 32 * (kWarps + 4);  // warps for rows; load, plan and two idle ones
constexpr int kCtlRegs = 72, kRowRegs = 216, kLaunchRegs = 168;        // 72 + 2 x 216 = 3 x 168
constexpr int kPieces = 4;                        // of 32 values, 128 bytes, a row
constexpr uint32_t kPiece = kKeys * 128u, kTile = kPieces * kPiece;
constexpr int kStages = 4;
constexpr uint64_t kDrainNs = 100000000ull;

template <int RW>
struct Shared {
  uint8_t ring[kStages][kTile];
  float o[kWarps][RW][128];
  float2 ml[kWarps][RW];
  unsigned path[RW][kTreeMaxNodes / 32];          // the nodes that a row sees, a bit each
  int used[RW], upto[RW];                         // upto: chains, keys that a row sees
  short up[kTreeMaxNodes];
  struct : Plan {
    uint64_t full[kStages], empty[kStages];
  } tail;
};

__device__ void load_role(const TreeParams& p, Plan* sh, uint64_t* full, uint64_t* empty, uint32_t ring0) {
  const int lane = threadIdx.x & 31;
  const int size = 1 << p.c.page_shift, box = min(size, kKeys), boxes = kKeys / box;
  // Halves of a row are read as a whole: what lies behind its end is filled with zeros.  boxes * parts <= 32.
  const int parts = p.dim > 64 ? 4 : 2, mine = lane / parts, part = lane - mine * parts;
  const bool active = mine < boxes;
  const int none = p.c.layers * p.c.pages * p.c.heads;  // a box there is filled with zeros
  const uint32_t skipped = tree_skipped(p);
  uint32_t ring = 0;
  bool ok = true;
  Seg g;
  for (uint32_t k = 0; ok && (ok = __all_sync(0xffffffffu, read_seg(p, sh, k, g))); ++k) {
    __syncwarp();
    if (lane == 0) free_seg(sh, k);
    const int* const table = g.row < 0 ? nullptr : p.c.table + static_cast<long long>(g.row) * p.c.max_pages;
    for (int j = g.t0; ok && j < g.t1; ++j) {
      const int pos = j * kKeys + mine * box, slot = pos & (size - 1);
      int at = none;
      if (active && table && pos < g.total) {
        const int page = table[pos >> p.c.page_shift];
        if (page >= 0 && page < p.c.pages) at = (p.layer * p.c.pages + page) * p.c.heads + g.head;
        else atomicOr(p.status, kStatusBadSeq);
      }
      for (int v = 0; v < 2; ++v, ++ring) {
        if (ring < skipped) continue;
        const uint32_t stage = ring % kStages;
        // (Warps whose wait for a stage ran out give it back all the same.  Filling it again would make its phases
        // other than its rounds, and the wait for copies at the end would miss some.)
        ok = __all_sync(0xffffffffu, wait_or_stop(p, sh, &empty[stage], ((ring / kStages) & 1u) ^ 1u));
        if (!ok) break;
        const uint32_t bar = smem_u32(&full[stage]);
        if (lane == 0) mbar_arrive_expect_tx(bar, parts * kPiece);
        __syncwarp();
        if (active)
          tma_load_3d(ring0 + stage * kTile + part * kPiece + mine * box * 128u, v ? &p.map_v : &p.map_k, bar, part * 32, slot, at);
      }
    }
  }
  if (lane == 0)  // what was asked for lands before the shared memory goes away
    for (uint32_t b = ring > kStages ? ring - kStages : skipped; b < ring; ++b)
      mbar_wait_drain(smem_u32(&full[b % kStages]), (b / kStages) & 1u, kDrainNs, p.status);
  __syncwarp();
}

template <int RW, bool kTwo>  // kTwo: rows of more than 64 values
__device__ void row_role(const TreeParams& p, Shared<RW>& s) {
  constexpr int RL = RW / 2, kDup = 16 / RL;      // a lane's rows; lanes that are left with the same one
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, half = lane >> 4, ls = lane & 15;
  const int own = half * RL + ls / kDup, units = p.dim / 4;
  // A lane's columns: 4 ls and 64 + 4 ls, where there are any.
  const bool some[2] = {ls < units, 16 + ls < units};
  uint32_t ring = 0;
  long long had_first = -1;                       // whose paths are in shared memory
  int had_row = -1, had_r0 = -1;
  Seg g;
  for (uint32_t k = 0;; ++k) {
    // All warps go on or leave together: the barriers below need all of them.  This one also says that all have
    // read what the last segment left in shared memory.
    if (!named_bar_and(1, kWarps * 32, read_seg(p, &s.tail, k, g))) break;
    if (lane == 0) free_seg(&s.tail, k);
    float4 q[RL][2];
#pragma unroll
    for (int i = 0; i < RL; ++i) {
      const int row = half * RL + i, r = g.r0 + row, node = r / p.group;
      const float* const from = static_cast<const float*>(p.q) + (g.first + node) * p.q_ld +
                                static_cast<long long>(g.head * p.group + r - node * p.group) * p.dim + 4 * ls;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        q[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row < g.nrows && some[c]) q[i][c] = *reinterpret_cast<const float4*>(from + 64 * c);
        if (p.negate) q[i][c] = make_float4(-q[i][c].x, -q[i][c].y, -q[i][c].z, -q[i][c].w);
      }
    }
    if (g.first != had_first || g.row != had_row || g.r0 != had_r0) {  // other heads of the same rows see the same
      had_first = g.first;
      had_row = g.row;
      had_r0 = g.r0;
      if (p.parents) {
        for (int j = tid; j < (g.row < 0 ? 0 : g.nodes); j += kWarps * 32) {
          const int u = p.parents[g.first + j];
          const bool odd = u < -2 || u >= j;
          if (odd) atomicOr(p.status, kStatusBadSeq);
          s.up[j] = static_cast<short>(odd ? -2 : u);
        }
        named_bar_sync(1, kWarps * 32);
      }
      if (tid < RW) {
        const int node = (g.r0 + tid) / p.group;
        bool used = g.row >= 0 && tid < g.nrows;
        s.upto[tid] = g.len + node + 1;
        if (p.parents) {
          used = used && s.up[node] >= -1;
          int j = used ? node : -1;
          for (int i = kTreeMaxNodes / 32 - 1; i >= 0; --i) {  // parents come before their children
            unsigned on = 0u;
            while (j >= 32 * i) {
              const int above = s.up[j];
              if (above >= -1) on |= 1u << (j & 31);
              j = above;
            }
            s.path[tid][i] = on;
          }
        }
        s.used[tid] = used;
      }
      named_bar_sync(1, kWarps * 32);
    }
    float m = -INFINITY, l = 0.f;                 // of row `own`
    float4 o[RL][2];
#pragma unroll
    for (int i = 0; i < RL; ++i) o[i][0] = o[i][1] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int t = g.t0; t < g.t1; ++t, ring += 2) {
      const int pos = t * kKeys + warp * 8;
      const bool masked = (t + 1) * kKeys > g.all;
      uint32_t stage = ring % kStages;
      const uint32_t chunk = (ls >> 3) * kPiece + warp * 1024u;
      wait(p, &s.tail, &s.tail.full[stage], (ring / kStages) & 1u);
      float z[8];
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) {
        const uint8_t* const at = s.ring[stage] + chunk + kk * 128 + (((ls & 7) ^ kk) << 4);
        const float4 f0 = *reinterpret_cast<const float4*>(at);
        float4 f1 = make_float4(0.f, 0.f, 0.f, 0.f);
        if (kTwo) f1 = *reinterpret_cast<const float4*>(at + 2 * kPiece);
        float v[RL];
#pragma unroll
        for (int i = 0; i < RL; ++i) {
          float2 a = mul2(make_float2(f0.x, f0.y), make_float2(q[i][0].x, q[i][0].y));
          a = fma2(make_float2(f0.z, f0.w), make_float2(q[i][0].z, q[i][0].w), a);
          if (kTwo) {
            a = fma2(make_float2(f1.x, f1.y), make_float2(q[i][1].x, q[i][1].y), a);
            a = fma2(make_float2(f1.z, f1.w), make_float2(q[i][1].z, q[i][1].w), a);
          }
          v[i] = a.x + a.y;
        }
        // Lanes whose bit is set go on with the upper half of the rows, the others with the lower.
#pragma unroll
        for (int n = RL / 2, bit = 8; bit > 0; bit >>= 1, n >>= 1) {
          const bool up = ls & bit;
          if (n > 0) {
#pragma unroll
            for (int i = 0; i < n; ++i) {
              const float give = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
              v[i] = keep + __shfl_xor_sync(0xffffffffu, give, bit);
            }
          } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], bit);
          }
        }
        z[kk] = v[0];
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&s.tail.empty[stage]));
      unsigned seen = 0xffu;                      // a bit a key, of row `own`
      if (masked) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
          const int j = pos + kk - g.len;
          bool on = s.used[own] && pos + kk < g.total;
          if (on && j >= 0) on = p.parents ? s.path[own][j >> 5] >> (j & 31) & 1u : pos + kk < s.upto[own];
          if (!on) {
            z[kk] = -INFINITY;
            seen &= ~(1u << kk);
          }
        }
      }
      const float now = fmaxf(m, fmax3(fmax3(z[0], z[1], z[2]), fmax3(z[3], z[4], z[5]), fmaxf(z[6], z[7])));
      const float base = tree_base(p, now);
      if (__any_sync(0xffffffffu, now > m)) {
        const float c = m == -INFINITY ? 0.f : exp2f(tree_base(p, m) - base);
        l *= c;
        m = now;
#pragma unroll
        for (int i = 0; i < RL; ++i) {
          const float ci = __shfl_sync(0xffffffffu, c, half * 16 + i * kDup);
          const float2 c2 = make_float2(ci, ci);
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float2 lo = mul2(make_float2(o[i][y].x, o[i][y].y), c2), hi = mul2(make_float2(o[i][y].z, o[i][y].w), c2);
            o[i][y] = make_float4(lo.x, lo.y, hi.x, hi.y);
          }
        }
      }
      float w[8];
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) w[kk] = seen >> kk & 1u ? exp2f(fmaf(z[kk], p.scale, -base)) : 0.f;
      l += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
      stage = (ring + 1) % kStages;
      wait(p, &s.tail, &s.tail.full[stage], ((ring + 1) / kStages) & 1u);
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) {
        const uint8_t* const at = s.ring[stage] + chunk + kk * 128 + (((ls & 7) ^ kk) << 4);
        const float4 f0 = *reinterpret_cast<const float4*>(at);
        float4 f1 = make_float4(0.f, 0.f, 0.f, 0.f);
        if (kTwo) f1 = *reinterpret_cast<const float4*>(at + 2 * kPiece);
#pragma unroll
        for (int i = 0; i < RL; ++i) {
          const float wk = __shfl_sync(0xffffffffu, w[kk], half * 16 + i * kDup);
          if (masked && !(__shfl_sync(0xffffffffu, seen, half * 16 + i * kDup) >> kk & 1u)) continue;  // it may be anything
          const float2 w2 = make_float2(wk, wk);
          const float2 a = fma2(make_float2(f0.x, f0.y), w2, make_float2(o[i][0].x, o[i][0].y));
          const float2 b = fma2(make_float2(f0.z, f0.w), w2, make_float2(o[i][0].z, o[i][0].w));
          o[i][0] = make_float4(a.x, a.y, b.x, b.y);
          if (kTwo) {
            const float2 c = fma2(make_float2(f1.x, f1.y), w2, make_float2(o[i][1].x, o[i][1].y));
            const float2 d = fma2(make_float2(f1.z, f1.w), w2, make_float2(o[i][1].z, o[i][1].w));
            o[i][1] = make_float4(c.x, c.y, d.x, d.y);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&s.tail.empty[stage]));
    }
    // The warps' parts of the keys meet.
    if (ls % kDup == 0) s.ml[warp][own] = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < RL; ++i)
#pragma unroll
      for (int c = 0; c < 2; ++c) *reinterpret_cast<float4*>(&s.o[warp][half * RL + i][64 * c + 4 * ls]) = o[i][c];
    named_bar_sync(1, kWarps * 32);
    const bool whole = g.t0 == 0 && g.t1 == g.nt;
    for (int x = tid; x < g.nrows * units; x += kWarps * 32) {
      // Lanes side by side: a row's columns, or of pieces a column's rows, as each lies in memory.
      const int row = whole ? x / units : x % g.nrows, c = whole ? x - row * units : x / g.nrows;
      float M = -INFINITY, sum = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s.ml[w][row].x);
      const float base = tree_base(p, M);
      for (int w = 0; w < kWarps; ++w) {
        const float2 ml = s.ml[w][row];
        if (ml.y == 0.f) continue;                // nothing seen
        const float f = ml.x == -INFINITY ? 1.f : exp2f(tree_base(p, ml.x) - base);  // a sum without a maximum is NaN
        const float4 b = *reinterpret_cast<const float4*>(&s.o[w][row][c * 4]);
        sum = fmaf(ml.y, f, sum);
        a = make_float4(fmaf(b.x, f, a.x), fmaf(b.y, f, a.y), fmaf(b.z, f, a.z), fmaf(b.w, f, a.w));
      }
      if (!s.used[row]) {
        sum = 0.f;
        a = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      if (whole) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const long long to = tree_out_row(p, g.first, g.head, g.r0 + row);
        *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to * p.dim + c * 4) =
            make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv);
        if (c == 0) p.lse[to] = tree_lse(p, M, sum);
      } else {
        float* const part = tree_part(p, blockIdx.x, g.slot);
        reinterpret_cast<float4*>(part)[static_cast<long long>(c + 1) * p.part_rows + row] = a;
        if (c == 0) reinterpret_cast<float2*>(part)[row] = make_float2(M, sum);
      }
    }
  }
}

template <int RW, bool kTwo>
__global__ void __launch_bounds__(kThreads, 1) tree_fp32_kernel(const __grid_constant__ TreeParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  Shared<RW>& s = *reinterpret_cast<Shared<RW>*>(smem);
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    plan_init(&s.tail, 1 + kWarps);
    for (int i = 0; i < kStages; ++i) {
      mbar_init(smem_u32(&s.tail.full[i]), 1);
      mbar_init(smem_u32(&s.tail.empty[i]), kWarps);
    }
    fence_barrier_init();
  }
  const Range range = plan_cut<kThreads>(p, &s.tail);  // has barriers
  chain_trigger();  // every CTA of this launch is resident: the next kernel's cannot take their place
  if (warp < kWarps) {
    if (RW == 16 && kTwo) regs_increase<kRowRegs>();
    row_role<RW, kTwo>(p, s);
  } else {
    if (RW == 16 && kTwo) regs_decrease<kCtlRegs>();
    if (warp == kWarps) load_role(p, &s.tail, s.tail.full, s.tail.empty, smem_u32(s.ring));
    else if (warp == kWarps + 1 && (threadIdx.x & 31) == 0) plan_role(p, &s.tail, range);
    __syncwarp();
  }
  __syncthreads();
}

// Joins the pieces of the items that lie in several CTAs' ranges, in order: blocks x have those of the item that
// CTA x began.  A thread has 16 values of a row; where there are many pieces, several threads share them.
// (Where a block of 32 threads' work each looked for the item itself, 16 trees of 64 nodes took 178 us instead of 130.)
constexpr int kJoinThreads = 256, kJoinParts = 8, kJoinWide = 4;  // pieces of four values a thread
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <bool kBf16>
__global__ void __launch_bounds__(kJoinThreads) tree_join_kernel(const __grid_constant__ TreeParams p) {
  __shared__ float s_top[kJoinThreads], s_sum[kJoinThreads];
  __shared__ float4 s_o[kJoinWide][kJoinThreads];
  chain_wait();
  const TreeJoin it = p.joins[blockIdx.x];
  const int units = p.dim / 4, all = it.rows * ((units + kJoinWide - 1) / kJoinWide), stride = p.part_rows;
  const int shift = it.pieces <= 4 ? 0 : it.pieces <= 8 ? 1 : it.pieces <= 16 ? 2 : 3;  // 2^shift threads share
  const int width = kJoinThreads >> shift, mine = threadIdx.x / width, own = threadIdx.x % width, step = 1 << shift;
  auto piece = [&](int c) { return tree_part(p, blockIdx.x + c, c == 0 ? it.slot : 0); };  // the first item of those behind
  for (int i0 = blockIdx.y * width; i0 < all; i0 += width * gridDim.y) {
    const int i = min(i0 + own, all - 1), x = i / it.rows * kJoinWide, r = i % it.rows;  // lanes side by side: rows that are
    float m = -INFINITY, l = 0.f;
    float4 o[kJoinWide];
#pragma unroll
    for (int y = 0; y < kJoinWide; ++y) o[y] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c = mine; c < it.pieces; c += 4 * step) {
      float top[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) top[y] = c + y * step < it.pieces ? piece(c + y * step)[2 * r] : -INFINITY;
#pragma unroll
      for (int y = 0; y < 4; ++y) m = fmaxf(m, top[y]);
    }
    if (shift) {
      s_top[threadIdx.x] = m;
      __syncthreads();
      for (int w = 0; w < step; ++w) m = fmaxf(m, s_top[w * width + own]);
    }
    const float base = tree_base(p, m);
    for (int c = mine; c < it.pieces; c += 2 * step) {
      float2 ml[2];
      float4 f[2][kJoinWide];
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const bool in = c + z * step < it.pieces;
        const float* const at = piece(in ? c + z * step : c);
        ml[z] = in ? *reinterpret_cast<const float2*>(at + 2 * r) : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int y = 0; y < kJoinWide; ++y)
          if (x + y < units) f[z][y] = *reinterpret_cast<const float4*>(at + (static_cast<long long>(x + y + 1) * stride + r) * 4);
      }
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        if (ml[z].y == 0.f) continue;
        const float k = ml[z].x == -INFINITY ? 1.f : exp2f(tree_base(p, ml[z].x) - base);  // a sum without a maximum is NaN
        l = fmaf(ml[z].y, k, l);
#pragma unroll
        for (int y = 0; y < kJoinWide; ++y)
          o[y] = make_float4(fmaf(f[z][y].x, k, o[y].x), fmaf(f[z][y].y, k, o[y].y), fmaf(f[z][y].z, k, o[y].z),
                             fmaf(f[z][y].w, k, o[y].w));
      }
    }
    if (shift) {
      s_sum[threadIdx.x] = l;
#pragma unroll
      for (int y = 0; y < kJoinWide; ++y) s_o[y][threadIdx.x] = o[y];
      __syncthreads();
      if (mine == 0)
        for (int w = 1; w < step; ++w) {
          l += s_sum[w * width + own];
#pragma unroll
          for (int y = 0; y < kJoinWide; ++y) {
            const float4 f = s_o[y][w * width + own];
            o[y] = make_float4(o[y].x + f.x, o[y].y + f.y, o[y].z + f.z, o[y].w + f.w);
          }
        }
    }
    if (mine == 0 && i0 + own < all) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const long long row = tree_out_row(p, it.first, it.head, it.r0 + r), to = row * p.dim + x * 4;
#pragma unroll
      for (int y = 0; y < kJoinWide; ++y) o[y] = make_float4(o[y].x * inv, o[y].y * inv, o[y].z * inv, o[y].w * inv);
      if (kBf16) {
#pragma unroll
        for (int y = 0; y < kJoinWide; y += 2)  // values come in eights
          if (x + y < units)
            st16(static_cast<__nv_bfloat16*>(p.out) + to + 4 * y,
                 make_uint4(pack(o[y].x, o[y].y), pack(o[y].z, o[y].w), pack(o[y + 1].x, o[y + 1].y), pack(o[y + 1].z, o[y + 1].w)));
      } else {
#pragma unroll
        for (int y = 0; y < kJoinWide; ++y)
          if (x + y < units) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to + 4 * y) = o[y];
      }
      if (x == 0) p.lse[row] = tree_lse(p, m, l);
    }
  }
}

}  // namespace

cudaError_t launch_tree_join(const TreeParams& p, cudaStream_t s) {
  const int parts = (p.part_rows * ((p.dim + 4 * kJoinWide - 1) / (4 * kJoinWide)) + kJoinThreads - 1) / kJoinThreads;
  return launch_chained(p.bf16 ? tree_join_kernel<true> : tree_join_kernel<false>,
                        dim3(p.sms - 1, parts < kJoinParts ? parts : kJoinParts), dim3(kJoinThreads), 0, s, p);
}

cudaError_t launch_tree_fp32(const TreeParams& p, cudaStream_t s) {
  if (p.item_rows == 4 && p.dim > 64) tree_fp32_kernel<4, true><<<p.sms, kThreads, sizeof(Shared<4>), s>>>(p);
  else if (p.item_rows == 4) tree_fp32_kernel<4, false><<<p.sms, kThreads, sizeof(Shared<4>), s>>>(p);
  else if (p.dim > 64) tree_fp32_kernel<16, true><<<p.sms, kThreads, sizeof(Shared<16>), s>>>(p);
  else tree_fp32_kernel<16, false><<<p.sms, kThreads, sizeof(Shared<16>), s>>>(p);
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? e : launch_tree_join(p, s);
}

void tree_sizes(TreeParams* p) {
  if (p->bf16) {
    p->tile_rows = tree_tile_rows(p->group);
    p->q_rows = tree_query_rows(p->group);
    p->item_rows = 2 * p->tile_rows;
    p->key_shift = 7;
    // (1, 3, 5, 8 and 12: 32 trees 90, 70, 71, 71 and 73 us, prompts 403, 369, 370, 376 and 383.)
    p->over = 4;
  } else {
    // Rows of an entry on average: where they are few, less is computed for nobody.
    p->item_rows = p->N * p->group <= 4LL * p->n ? 4 : 16;
    p->key_shift = 6;
    p->over = 2;  // (4 and 8: prompts of 1500 tokens 185 and 208 us instead of 173)
  }
  p->part_rows = static_cast<int>(p->N * p->group < p->item_rows ? p->N * p->group : p->item_rows);
}

cudaError_t setup_tree_kernels() {
  static_assert(sizeof(Shared<16>) <= 227 * 1024, "shared memory");
  cudaError_t e = cudaSuccess;
  for (void (*kernel)(TreeParams) : {tree_fp32_kernel<4, false>, tree_fp32_kernel<4, true>})
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Shared<4>));
  for (void (*kernel)(TreeParams) : {tree_fp32_kernel<16, false>, tree_fp32_kernel<16, true>})
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Shared<16>));
  if (e != cudaSuccess) return e;
  cudaFuncAttributes fa;
  if ((e = cudaFuncGetAttributes(&fa, tree_fp32_kernel<16, true>)) != cudaSuccess) return e;
  // The split of registers between the roles waits forever unless the launch has just that many.
  if (fa.numRegs != kLaunchRegs || fa.maxThreadsPerBlock < kThreads) return cudaErrorInvalidConfiguration;
  return setup_tree_mma_kernels();
}

}  // namespace mls
