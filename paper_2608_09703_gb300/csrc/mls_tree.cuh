// What the tree-attention kernels share: the entries of a call, and how its work is cut into equal ranges.
//
// Items are (entry, item_rows of its rows, key/value head); the rows of an entry are its nodes times the query
// heads of one key/value head (node-major).  Lengths are known on the device only, so CTAs cut the work there: the
// key tiles of all items, and `over` units more for each item's beginning and end, are numbered, and CTA c of G takes
// the c-th of G equal ranges, which may begin and end inside an item.  Pieces of an item that lies in several
// ranges go to the workspace, and a second kernel joins them, as the first of the CTAs wrote it down.  Work is
// even over the card whatever the lengths are, and a captured graph follows them.
#pragma once

#include "mls_device.cuh"
#include "mls_kernels.h"

namespace mls {

constexpr float kLn2 = 0.6931471805599453f;

// Weights are 2^(scale z - base) with base = scale m rounded, m a maximum: what they are brought to, and what lse
// adds, is that same number.
__device__ __forceinline__ float tree_base(const TreeParams& p, float m) { return m == -INFINITY ? 0.f : __fmul_rn(m, p.scale); }
__device__ __forceinline__ float tree_lse(const TreeParams& p, float m, float sum) {
  return sum == 0.f ? -INFINITY : (tree_base(p, m) + log2f(sum)) * kLn2;
}

// What an entry of a call is: its nodes [first, first + nodes) of the packed ones, its row of the
// table and the tokens cached there.  What does not fit the cache is an entry of unused nodes.
struct Entry {
  int nodes, row, len;
  long long first;
};
__device__ __forceinline__ Entry tree_entry(const TreeParams& p, int i, int* status) {
  Entry e;
  const long long a = p.start[i], b = p.start[i + 1];
  e.row = p.seqs ? p.seqs[i] : i;
  const bool known = e.row >= 0 && e.row < p.c.seqs;
  e.len = known ? p.c.len[e.row] : 0;             // does not wait for what start says
  bool bad = a < 0 || b < a || b > p.N;
  e.first = a;
  e.nodes = bad ? 0 : static_cast<int>(b - a);
  if (e.nodes == 0) {
    e.len = 0;
  } else if (!known || (p.parents && e.nodes > kTreeMaxNodes) || e.len < 0 ||
             static_cast<long long>(e.len) + e.nodes > (static_cast<long long>(p.c.max_pages) << p.c.page_shift)) {
    bad = true;
    e.row = -1;
    e.len = 0;
  }
  if (bad) atomicOr(status, kStatusBadSeq);
  return e;
}

// A run of items of an entry that have as many key tiles each: those of rows r0, r0 + item_rows, ...
struct Run {
  int r0, rows, count, total, nt;                 // rows and keys of the first
};
__device__ __forceinline__ Run tree_run(const TreeParams& p, const Entry& en, int r0) {
  Run u;
  const int all = en.nodes * p.group;
  u.r0 = r0;
  u.rows = min(all - r0, p.item_rows);
  u.total = en.len + (r0 + u.rows - 1) / p.group + 1;
  u.nt = ((u.total - 1) >> p.key_shift) + 1;
  // An item of nt tiles has its last row below `most`.
  const long long most = ((static_cast<long long>(u.nt) << p.key_shift) - en.len) * p.group;
  u.count = most >= all ? (all - r0 + p.item_rows - 1) / p.item_rows : static_cast<int>(most - r0) / p.item_rows;
  return u;
}
__device__ inline long long entry_units(const TreeParams& p, const Entry& en) {
  long long sum = 0;
  for (int r0 = 0; r0 < en.nodes * p.group;) {
    const Run u = tree_run(p, en, r0);
    sum += static_cast<long long>(u.count) * (p.over + u.nt);
    r0 += u.count * p.item_rows;
  }
  return sum * p.c.heads;
}

// A piece of an item, for every role: rows [r0, r0 + nrows) of an entry and head, key tiles [t0, t1) of nt.
struct Seg {
  long long first;                                // of the entry's nodes
  int nodes, row, len;                            // its nodes, row of the table (-1: none takes part) and cached tokens
  int head, r0, nrows, t0, t1, nt;                // t0 = t1: the end
  int total;                                      // keys of the item: cached tokens and nodes up to its last
  int all;                                        // keys that every row sees
  int slot;                                       // of the CTA's two in the workspace
  int solo, other;                                // bf16: 1, 2: of a couple, with `other` tiles in the other one
};
constexpr int kSegs = 4;
constexpr int kSoloTiles = 8;                     // at most, of a couple's segments
// In shared memory.
struct Plan {
  uint64_t seg_full[kSegs], seg_empty[kSegs];
  Seg seg[kSegs];
  Entry en0;                                      // the range's first entry, its number and first unit
  long long scan[12], base0;                      // of at most 12 warps
  int e0, abort;
};

__device__ __forceinline__ bool wait(const TreeParams& p, Plan* sh, uint64_t* bar, uint32_t parity) {
  return mbar_wait(smem_u32(bar), parity, &sh->abort, p.status);
}
// As `wait`, for one who is to stop where another gave up, even if what it waits for came.
__device__ __forceinline__ bool wait_or_stop(const TreeParams& p, Plan* sh, uint64_t* bar, uint32_t parity) {
  return wait(p, sh, bar, parity) && !*static_cast<volatile int*>(&sh->abort);
}
// Test hook (off unless the host sets it): stages at the beginning that each CTA brings nothing for, so that the wait for
// them runs out.  (Each: which CTAs have tiles depends on the lengths.)
__device__ __forceinline__ uint32_t tree_skipped(const TreeParams& p) { return p.test_stall != 0; }
__device__ inline void plan_init(Plan* sh, int readers) {
  sh->abort = 0;
  for (int k = 0; k < kSegs; ++k) {
    mbar_init(smem_u32(&sh->seg_full[k]), 1);
    mbar_init(smem_u32(&sh->seg_empty[k]), readers);
  }
}

// The CTA's range [lo, hi) of units, of `each` a CTA.  All threads: each adds up a run of entries.  Two barriers.
struct Range {
  long long lo, hi, each;
};
template <int kThreads>
__device__ Range plan_cut(const TreeParams& p, Plan* sh) {
  static_assert(kThreads <= 12 * 32, "Plan::scan");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int chunk = (p.n + kThreads - 1) / kThreads;
  const int i0 = min(tid * chunk, p.n), i1 = min(i0 + chunk, p.n);
  long long mine = 0;
  for (int i = i0; i < i1; ++i) mine += entry_units(p, tree_entry(p, i, p.status));
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) sh->scan[warp] = upto;
  __syncthreads();
  long long before = upto - mine, units = 0;
  for (int x = 0; x < kThreads / 32; ++x) {
    if (x < warp) before += sh->scan[x];
    units += sh->scan[x];
  }
  Range r;
  r.each = (units + gridDim.x - 1) / gridDim.x;
  r.lo = min(blockIdx.x * r.each, units);
  r.hi = min(r.lo + r.each, units);
  if (r.lo < r.hi && before <= r.lo && r.lo < before + mine) {
    long long at = before;
    for (int i = i0; i < i1; ++i) {
      const Entry en = tree_entry(p, i, p.status);
      const long long u = entry_units(p, en);
      if (at <= r.lo && r.lo < at + u) {
        sh->en0 = en;
        sh->e0 = i;
        sh->base0 = at;
      }
      at += u;
    }
  }
  __syncthreads();
  return r;
}

// One thread: writes down the segments of the range, and what begins there and goes on in other CTAs'.  Two short
// ones of about as many tiles that follow one another make a couple, where the kernel works on such side by side
// (224 trees of 5 nodes, 16 heads: 164 us without, 116 with; 256 single tokens over up to 1000: 362 and 277).
__device__ inline void plan_role(const TreeParams& p, Plan* sh, const Range& range) {
  uint32_t k = 0;
  bool first = true;
  TreeJoin join = {};
  auto slot = [&](uint32_t i) -> Seg* {
    return wait(p, sh, &sh->seg_empty[i % kSegs], ((i / kSegs) & 1u) ^ 1u) ? &sh->seg[i % kSegs] : nullptr;
  };
  auto publish = [&] { mbar_arrive(smem_u32(&sh->seg_full[k++ % kSegs])); };
  int held = 0;                                   // tiles of the k-th, written down, that waits for one to make a couple with
  long long at = range.lo;
  if (at < range.hi) {
    Entry en = sh->en0;
    int e = sh->e0;
    long long v = at - sh->base0;                 // units into the run
    Run u = {};
    bool some = en.nodes > 0;
    if (some) u = tree_run(p, en, 0);
    while (at < range.hi) {
      while (!some || v >= static_cast<long long>(u.count) * (u.nt + p.over) * p.c.heads) {
        int r0 = 0;
        if (some) {
          v -= static_cast<long long>(u.count) * (u.nt + p.over) * p.c.heads;
          r0 = u.r0 + u.count * p.item_rows;
        }
        if (!some || r0 >= en.nodes * p.group) {
          en = tree_entry(p, ++e, p.status);
          some = en.nodes > 0;
          r0 = 0;
        }
        if (some) u = tree_run(p, en, r0);
      }
      // The item, and where in it: its rows come after those of all heads before.
      const int size = u.nt + p.over;
      // (In 32 bits where they do: a division of 64 is slow, and this is a thread's latency.)
      const long long item = v >> 31 ? v / size : static_cast<unsigned>(v) / static_cast<unsigned>(size);
      const int in = static_cast<int>(v - item * size);
      const int up = item >> 31 ? static_cast<int>(item / p.c.heads) : static_cast<int>(static_cast<unsigned>(item) / p.c.heads);
      const int head = static_cast<int>(item - static_cast<long long>(up) * p.c.heads), r0 = u.r0 + up * p.item_rows;
      const int end = static_cast<int>(min(static_cast<long long>(size), in + (range.hi - at)));
      at += end - in;
      v += end - in;
      const int t0 = max(in - p.over, 0), t1 = end - p.over;
      if (t1 <= t0) continue;                     // the range ends before the item's first tile
      Seg* const g = slot(held ? k + 1 : k);
      if (!g) break;
      g->first = en.first;
      g->nodes = en.nodes;
      g->row = en.row;
      g->len = en.len;
      g->head = head;
      g->r0 = r0;
      g->nrows = min(en.nodes * p.group - r0, p.item_rows);
      g->t0 = t0;
      g->t1 = t1;
      g->nt = u.nt;
      g->total = en.len + (r0 + g->nrows - 1) / p.group + 1;
      g->all = en.row < 0 ? 0 : p.parents ? en.len : en.len + r0 / p.group + 1;
      g->slot = first ? 0 : 1;
      g->solo = g->other = 0;
      first = false;
      MLS_CHECK(p.status, head < p.c.heads && g->nrows > 0 && g->nrows <= p.part_rows && t1 <= u.nt && (u.nt - 1) << p.key_shift < g->total &&
                              g->first + (r0 + g->nrows - 1) / p.group < p.N);
      if (t0 == 0 && t1 < u.nt) {                 // at = hi: the range ends after tile t1 of the item
        join.pieces = 1 + static_cast<int>((u.nt - t1 + range.each - 1) / range.each);
        join.slot = g->slot;
        MLS_CHECK(p.status, blockIdx.x + join.pieces <= gridDim.x);
        join.rows = g->nrows;
        join.first = static_cast<int>(en.first);
        join.r0 = r0;
        join.head = head;
      }
      const int n = t1 - t0;
      const bool may = p.bf16 && g->nrows <= p.tile_rows && n <= kSoloTiles;
      const bool couple = held && may && abs(n - held) <= p.over;
      if (couple) {
        sh->seg[k % kSegs].solo = 1;
        sh->seg[k % kSegs].other = n;
        g->solo = 2;
        g->other = held;
      }
      if (held) publish();
      held = may && !couple ? n : 0;
      if (!held) publish();
    }
    if (held) publish();
  }
  p.joins[blockIdx.x] = join;
  if (Seg* const g = slot(k)) {
    g->t0 = g->t1 = 0;
    publish();
  }
}
// The k-th segment for one of its readers (false: there is none, or a wait ran out).
__device__ __forceinline__ bool read_seg(const TreeParams& p, Plan* sh, uint32_t k, Seg& g) {
  if (!wait(p, sh, &sh->seg_full[k % kSegs], (k / kSegs) & 1u)) return false;
  g = sh->seg[k % kSegs];
  return g.t1 > g.t0;
}
__device__ __forceinline__ void free_seg(Plan* sh, uint32_t k) { mbar_arrive(smem_u32(&sh->seg_empty[k % kSegs])); }

// A piece's rows in the workspace: float2 [part_rows] of maximum and sum, float4 [dim / 4][part_rows].
__device__ __forceinline__ float* tree_part(const TreeParams& p, long long cta, int slot) {
  return p.part + (cta * 2 + slot) * p.part_rows * (p.dim + 4);
}
// Where an item's row goes in out [N * q_heads] and lse.
__device__ __forceinline__ int tree_out_row(const TreeParams& p, long long first, int head, int r) {
  const int node = r / p.group;
  return (static_cast<int>(first) + node) * p.q_heads + head * p.group + (r - node * p.group);
}

}  // namespace mls
