// Tree attention over a bf16 cache on the tensor cores (the operator: mls_tree.cu).
//
// The rows of a product are an entry's nodes times the query heads of one key/value head (node-major), 128 a
// tile.  S = Q K^T and O += P V run as tcgen05 MMAs of 128 rows and 128 keys; K and V come by TMA, a box a page
// (V in place as an MN-major operand), P goes back to TMEM as the A operand, over S.
// A CTA has two streams of a warpgroup, an S and an O accumulator each (512 columns of TMEM): the tensor cores
// work for one while the other takes its exponentials.  With more than 128 rows the streams have a row
// tile each and share the keys; with fewer they have the same rows, and every other key tile: what they
// hold is joined at the end, each warp reading the other stream's O in its own lanes.  Two short pieces of work with
// a row tile each are taken side by side, a stream each: what begins and ends one hides behind the other.
// Items are pairs of row tiles of an entry and key/value head, cut into ranges as mls_tree.cuh has it.
//
// Softmax in one pass: a running maximum per row, which moves only where weights would pass 2^8, so that O is
// rarely rescaled (a published technique: rescaling past a threshold only).  Scores, sums, maxima and O are fp32; P
// is rounded to bf16 for its product, as the tensor cores take operands of one type and V is bf16.  That moves each
// weight by 2^-9 on average, whatever its size: 1.5e-3 of out's norm, beside the 1.7e-3 of rounding out itself.
// Only tiles past the cached tokens look at masks.  Masked weights are 0, and so that 0 times what lies there is 0
// too, values behind the item's last node are cleared, and infinities and NaN among the nodes' values taken out of
// the product and added to the rows that do see them.
#include <cmath>

#include "mls_device.cuh"
#include "mls_kernels.h"
#include "mls_tree.cuh"
#include "mls_vec.cuh"

namespace mls {
namespace {

constexpr int kRows = 128, kKeys = 128;           // of a tile
constexpr int kThreads = 384;
constexpr int kCtlRegs = 88, kSoftmaxRegs = 208, kLaunchRegs = 168;  // 88 + 2 x 208 = 3 x 168
constexpr uint64_t kDrainNs = 100000000ull;
constexpr uint32_t kTmemCols = 512, kAccO = 256;  // S of stream w at 128 w, O at 256 + 128 w
constexpr float kGrow = 8.f;
constexpr int kMaxStages = 12;
constexpr uint32_t kSmem = 227 * 1024;

constexpr int kSegReaders = 3 + 8;                // load, MMA and query warp, eight of softmax
// Past the operands.  A warpgroup's `up` and `ml` share memory: parents are read before any sum is.
struct Tail : Plan {
  uint64_t full[kMaxStages], empty[kMaxStages], q_ready[2], q_free[2], s_full[2], p_ready[2][2], o_full[2], met, drain;
  union {
    short up[kTreeMaxNodes];
    float2 ml[kRows];
  } row[2];
  // By a segment's last two bits (streams are at most three segments apart): the last one with values taken out.
  int fix[4];
  uint32_t tmem_slot;
};
// DC: pieces of 64 values (128 bytes) of a row.  K and V tiles lie in atoms of 8 rows of 128 bytes; of rows of
// 128 values (kJoint) the two pieces' atoms alternate, so that one TMA box brings a page.
template <int DC, bool kJoint>
struct Layout {
  static constexpr uint32_t kTile = DC * kKeys * 128u;
  static constexpr int kStages = DC == 2 ? 5 : 12;
  static constexpr uint32_t kRing = 2 * kTile, kTail = kRing + kStages * kTile;
  static constexpr uint32_t kAtom = kJoint ? 2048u : 1024u;         // between atoms of rows
  static constexpr uint32_t kPiece = kJoint ? 1024u : kKeys * 128u; // between pieces
  static_assert(kTail + sizeof(Tail) <= kSmem, "shared memory");
  static_assert(!kJoint || DC == 2, "two pieces");
  // Where 16 bytes of a tile lie: row, and which of the row's (not swizzled).
  static __device__ __forceinline__ uint32_t at(int row, int c) {
    return (row >> 3) * kAtom + (row & 7) * 128u + (c >> 3) * kPiece + ((c & 7) << 4);
  }
};

// The order in which tiles are loaded, as the MMAs take them: for two row tiles K V K V ...; for two streams with n0
// and n1 steps of their own (a couple's, or every other tile of one segment) K K, then V of a step and K of the
// next for each stream in turn, as far as there are any.  Where V of step i lies then:
__device__ __forceinline__ uint32_t place_v(int n0, int n1, int w, int i) {
  const int a = i + w;                            // steps of the first stream that come before it
  return min(n1, 1) + 1 + min(a, n0) + min(a, n0 - 1) + min(i, n1) + min(i, max(n1 - 1, 0));
}

template <int DC, bool kJoint>
__device__ void load_role(const TreeParams& p, Tail* sh, uint32_t base) {
  using L = Layout<DC, kJoint>;
  const int lane = threadIdx.x & 31;
  const int size = 1 << p.c.page_shift, box = min(size, kKeys), boxes = kKeys / box;
  constexpr int kParts = kJoint ? 1 : DC;                     // boxes of a page
  const int mine = lane / kParts, part = lane - mine * kParts;  // this lane's box of a tile: boxes * kParts <= 32
  const bool active = mine < boxes;
  const int none = p.c.layers * p.c.pages * p.c.heads;        // a box there is filled with zeros
  const uint32_t dst = part * L::kPiece + mine * (box >> 3) * L::kAtom, skipped = tree_skipped(p);
  uint32_t ring = 0;
  bool ok = true;
  Seg g;
  for (uint32_t k = 0; ok && (ok = __all_sync(0xffffffffu, read_seg(p, sh, k, g))); ++k) {
    __syncwarp();
    if (lane == 0) free_seg(sh, k);
    const int n = g.t1 - g.t0;
    const bool pair = g.nrows > p.tile_rows;
    const int each = pair || g.solo ? 1 : 2, n0 = each == 1 ? n : (n + 1) / 2, n1 = pair ? 0 : g.solo ? g.other : n / 2;
    // What the second stream's tiles are of: the couple's other segment, or the same one, from its second tile on.
    int row = g.row, head = g.head, t0 = g.t0 + 1, total = g.total;
    if (g.solo) {
      Seg b;
      ok = __all_sync(0xffffffffu, read_seg(p, sh, ++k, b));
      row = b.row, head = b.head, t0 = b.t0, total = b.total;
      __syncwarp();
      if (lane == 0) free_seg(sh, k);
    }
#pragma unroll 1
    for (int x = 1; ok && (x >> 2) <= max(n0, n1); ++x) {  // K K, then V K V K of each step
      const bool second = x & 2, is_v = !(x & 1);
      const int i = (x >> 2) - is_v;
      if (i < 0 || i >= (second ? n1 : n0)) continue;
      const int pos = ((second ? t0 : g.t0) + i * each) * kKeys + mine * box, slot = pos & (size - 1);
      const int of = second ? row : g.row;
      int at = none;
      if (active && of >= 0 && pos < (second ? total : g.total)) {
        const int page = p.c.table[static_cast<long long>(of) * p.c.max_pages + (pos >> p.c.page_shift)];
        if (page >= 0 && page < p.c.pages) at = (p.layer * p.c.pages + page) * p.c.heads + (second ? head : g.head);
        else atomicOr(p.status, kStatusBadSeq);
      }
      if (ring < skipped) {
        ++ring;
        continue;
      }
      const uint32_t stage = ring % L::kStages, phase = (ring / L::kStages) & 1u;
      ok = __all_sync(0xffffffffu, wait(p, sh, &sh->empty[stage], phase ^ 1u));
      if (!ok) break;
      ++ring;
      const uint32_t bar = smem_u32(&sh->full[stage]), to = base + L::kRing + stage * L::kTile + dst;
      if (lane == 0) mbar_arrive_expect_tx(bar, L::kTile);
      __syncwarp();
      const CUtensorMap* const map = is_v ? &p.map_v : &p.map_k;
      if (active) {
        if (kJoint) tma_load_5d(to, map, bar, 0, 0, 0, slot >> 3, at);
        else tma_load_3d(to, map, bar, part * 64, slot, at);
      }
    }
  }
  if (lane == 0)  // what was asked for lands before the shared memory goes away
    for (uint32_t b = ring > L::kStages ? ring - L::kStages : skipped; b < ring; ++b)
      mbar_wait_drain(smem_u32(&sh->full[b % L::kStages]), (b / L::kStages) & 1u, kDrainNs, p.status);
  __syncwarp();
}

// One warp: queries of each stream's rows.  A TMA box has the heads of some nodes, in the order of the rows; nodes
// behind the entry's may come with it: their rows are nobody's.  Groups of more than a tile's rows are
// gathered, swizzled as TMA would.
template <int DC>
__device__ void query_role(const TreeParams& p, Tail* sh, uint32_t base) {
  constexpr int kWide = DC * 8, kStep = 32 / kWide;           // pieces of 16 bytes of a row, rows at a time
  const int lane = threadIdx.x & 31, c = lane % kWide;
  const int part = lane % DC, mine = lane / DC;               // this lane's box: at most 16 of DC pieces
  uint32_t loads[2] = {0, 0};
  bool ok = true;
  Seg g;
  for (uint32_t k = 0; ok && __all_sync(0xffffffffu, read_seg(p, sh, k, g)); ++k) {
    __syncwarp();
    if (lane == 0) free_seg(sh, k);
    const int n = g.t1 - g.t0;
    const bool pair = g.nrows > p.tile_rows;
    for (int w = 0; w < 2; ++w) {
      if (g.solo ? w != g.solo - 1 : !pair && w == 1 && n < 2) continue;
      ok = __all_sync(0xffffffffu, wait(p, sh, &sh->q_free[w], (loads[w] & 1u) ^ 1u));
      if (!ok) break;
      ++loads[w];
      const int row0 = g.r0 + (pair ? w * p.tile_rows : 0), last = g.r0 + g.nrows;
      const uint32_t bar = smem_u32(&sh->q_ready[w]), tile = base + w * DC * kRows * 128u;
      if (p.q_rows) {
        const int boxes = (min(last - row0, p.tile_rows) + p.q_rows - 1) / p.q_rows;
        if (lane == 0) mbar_arrive_expect_tx(bar, boxes * DC * p.q_rows * 128u);
        __syncwarp();
        if (mine < boxes)
          tma_load_3d(tile + part * (kRows * 128u) + mine * p.q_rows * 128u, &p.map_q, bar, part * 64, g.head * p.group,
                      static_cast<int>(g.first) + (row0 + mine * p.q_rows) / p.group);
        continue;
      }
      int r = row0 + lane / kWide, t = r / p.group, h = r - t * p.group;
      const __nv_bfloat16* const q = static_cast<const __nv_bfloat16*>(p.q) + g.first * p.q_ld +
                                     static_cast<long long>(g.head) * p.group * p.dim + c * 8;
      uint32_t to = tile + (c >> 3) * (kRows * 128u) + (lane / kWide) * 128u;
#pragma unroll 4
      for (int i = lane / kWide; i < kRows; i += kStep) {
        const bool in = r < last && c * 8 < p.dim;
        cp_async_16(to + (((c & 7) ^ (i & 7)) << 4), in ? q + t * p.q_ld + static_cast<long long>(h) * p.dim : p.q, in);
        to += kStep * 128u;
        r += kStep;
        h += kStep;
        while (h >= p.group) {
          h -= p.group;
          ++t;
        }
      }
      cp_async_wait_all();
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    }
  }
  if (lane == 0)
    for (int w = 0; w < 2; ++w)
      if (loads[w]) mbar_wait_drain(smem_u32(&sh->q_ready[w]), (loads[w] - 1) & 1u, kDrainNs, p.status);
  __syncwarp();
}

// One warp, which runs as one (all of its lanes wait) down to the elected lane that issues.
template <int DC, bool kJoint>
__device__ void mma_role(const TreeParams& p, Tail* sh, uint32_t base, uint32_t tmem) {
  using L = Layout<DC, kJoint>;
  constexpr uint32_t kNegateA = 1u << 13;
  const uint32_t idesc_s = make_idesc(kRows, kKeys, false, false, false) | (p.negate ? kNegateA : 0u);
  const int dn = (p.dim + 15) & ~15;
  const uint32_t idesc_o = make_idesc(kRows, dn, false, false, true);
  const int ks = dn / 16, lane = threadIdx.x & 31;
  // A place in the ring, and which round.
  struct Place {
    uint32_t stage, phase;
    __device__ __forceinline__ Place next() const {
      return stage + 1 == L::kStages ? Place{0, phase ^ 1u} : Place{stage + 1, phase};
    }
  };
  Place at = {0, 0};
  uint32_t q_par = 0, p_par = 0;  // a bit a stream
  bool ok = true;
  auto ready = [&](uint64_t* bar, uint32_t parity) {
    ok = ok && __all_sync(0xffffffffu, wait(p, sh, bar, parity));
    tc_fence_after();
    return ok;
  };
  Seg g;
  for (uint32_t k = 0; ok && __all_sync(0xffffffffu, read_seg(p, sh, k, g)); ++k) {
    __syncwarp();
    if (lane == 0) free_seg(sh, k);
    const int n = __shfl_sync(0xffffffffu, g.t1 - g.t0, 0);
    const bool pair = __shfl_sync(0xffffffffu, g.nrows, 0) > p.tile_rows;
    // S of stream w from the K tile at `from`, which it is the last to read or not.
    auto scores = [&](int w, const Place& from, bool last, bool done) {
      const uint64_t a = make_sdesc(base + w * L::kTile, 16), b = make_sdesc(base + L::kRing + from.stage * L::kTile, 16, L::kAtom);
      if (elect_one()) {
#pragma unroll
        for (int x = 0; x < DC * 4; ++x)
          if (x < ks)
            mma_issue<false>(tmem + w * kKeys, a + (x >> 2) * (kRows * 128 / 16) + (x & 3) * 2,
                             b + (x >> 2) * (L::kPiece / 16) + (x & 3) * 2, idesc_s, x > 0);
        mma_commit(smem_u32(&sh->s_full[w]));
        if (done) mma_commit(smem_u32(&sh->empty[from.stage]));
        if (last) mma_commit(smem_u32(&sh->q_free[w]));
      }
      __syncwarp();
    };
    // O of stream w from the V tile at `from`, its P in two halves.
    auto values = [&](int w, const Place& from, bool first, bool last, bool done) {
      const uint64_t b = make_sdesc(base + L::kRing + from.stage * L::kTile, L::kPiece, L::kAtom);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (!ready(&sh->p_ready[w][h], (p_par >> w) & 1u)) return;
        if (elect_one()) {
#pragma unroll
          for (int x = 4 * h; x < 4 * h + 4; ++x)
            mma_issue_ts(tmem + kAccO + w * 128, tmem + w * kKeys + x * 8, b + x * (2 * L::kAtom / 16), idesc_o,
                         !first || x > 0);
          if (h == 1) {
            if (done) mma_commit(smem_u32(&sh->empty[from.stage]));
            if (last) mma_commit(smem_u32(&sh->o_full[w]));
          }
        }
        __syncwarp();
      }
      p_par ^= 1u << w;
    };
    if (pair) {  // K | V K | V K ... each for both
      for (int w = 0; ok && w < 2; ++w) {
        if (!ready(&sh->q_ready[w], (q_par >> w) & 1u)) break;
        if (w == 0 && !ready(&sh->full[at.stage], at.phase)) break;
        scores(w, at, n == 1, w == 1);
      }
      q_par ^= 3u;
      at = at.next();
      for (int i = 0; ok && i < n; ++i) {
        const Place v = at, key = at.next();
        const bool more = i + 1 < n;
        if (!ready(&sh->full[v.stage], v.phase)) break;
        for (int w = 0; ok && w < 2; ++w) {
          values(w, v, i == 0, !more, w == 1);
          if (!more) continue;
          if (w == 0 && !ready(&sh->full[key.stage], key.phase)) break;
          if (ok) scores(w, key, i + 2 == n, w == 1);
        }
        at = more ? key.next() : key;
      }
      continue;
    }
    // K K | V K | V K ... of either stream in turn.
    const bool solo = __shfl_sync(0xffffffffu, g.solo, 0) != 0;
    const int n0 = solo ? n : (n + 1) / 2, n1 = solo ? __shfl_sync(0xffffffffu, g.other, 0) : n / 2;
    if (solo) {  // the stream's other segment: all there is to know of it is here
      if (!(ok = __all_sync(0xffffffffu, wait(p, sh, &sh->seg_full[(k + 1) % kSegs], ((k + 1) / kSegs) & 1u)))) break;
      ++k;
      if (lane == 0) free_seg(sh, k);
    }
    for (int i = -1; ok && i < max(n0, n1); ++i)
      for (int w = 0; ok && w < 2; ++w) {
        const int steps = w ? n1 : n0;
        if (i >= steps || (i < 0 && steps == 0)) continue;
        if (i >= 0) {
          if (!ready(&sh->full[at.stage], at.phase)) break;
          values(w, at, i == 0, i + 1 == steps, true);
          at = at.next();
        } else {
          if (!ready(&sh->q_ready[w], (q_par >> w) & 1u)) break;
          q_par ^= 1u << w;
        }
        if (!ok || i + 1 >= steps) continue;
        if (!ready(&sh->full[at.stage], at.phase)) break;
        scores(w, at, i + 2 == steps, true);
        at = at.next();
      }
  }
  // Every MMA that the elected lane issued has finished before TMEM is released.
  if (elect_one()) mma_commit(smem_u32(&sh->drain));
  __syncwarp();
  mbar_wait_drain(smem_u32(&sh->drain), 0, kDrainNs, p.status);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Halves of a word that are infinite or NaN.
__device__ __forceinline__ bool odd_lo(uint32_t w) { return (w & 0x7f80u) == 0x7f80u; }
__device__ __forceinline__ bool odd_hi(uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ bool odd_any(const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) odd |= odd_lo(w[i]) || odd_hi(w[i]);
  return odd;
}

// What a row sees past the cached tokens: the nodes up to its own, or those on its path.
struct Sight {
  unsigned path[kTreeMaxNodes / 32];
  int len, upto;                                  // keys before `upto` where there is no path
  bool tree, used;
  // Truth of keys [k, k + 32), a bit each.
  __device__ __forceinline__ unsigned bits(int k) const {
    if (!used) return 0u;
    if (!tree) {
      const int n = upto - k;
      return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
    }
    const int j = k - len;                        // node of the first
    if (j <= -32) return 0xffffffffu;
    const int word = j >> 5, shift = j & 31;      // rounds down
    unsigned lo = word < 0 ? 0xffffffffu : 0u, hi = 0u;
#pragma unroll
    for (int i = 0; i < kTreeMaxNodes / 32; ++i) {
      if (i == word) lo = path[i];
      if (i == word + 1) hi = path[i];
    }
    return __funnelshift_r(lo, hi, shift);
  }
};

template <int DC, bool kJoint>
__device__ void softmax_role(const TreeParams& p, Tail* sh, uint32_t base, uint32_t tmem, int w) {
  using L = Layout<DC, kJoint>;
  const int tid = threadIdx.x & 127, quad = tid >> 5, lane = tid & 31;
  const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
  const uint32_t ts = tmem + lanes + w * kKeys, to = tmem + lanes + kAccO + w * 128;
  const __nv_bfloat16* const V = reinterpret_cast<const __nv_bfloat16*>(p.c.v);
  const int mask = (1 << p.c.page_shift) - 1;
  uint32_t ring = 0, couple = 0, s_par = 0, o_par = 0, met = 0;
  auto meet = [&] {                               // both streams (a wait with a limit, unlike a barrier)
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sh->met));
    wait(p, sh, &sh->met, met);
    met ^= 1u;
  };
  Sight see;
  long long had_first = -1;                       // whose `see` this is
  int had_row = -1, had_r0 = -1;
  Seg g;
  for (uint32_t k = 0;; ++k) {
    const int seg = static_cast<int>(k) + 1;
    // All of a warpgroup go on or leave together: the barriers below need all of them.
    if (!named_bar_and(1 + w, kRows, read_seg(p, sh, k, g))) break;
    if (lane == 0) free_seg(sh, k);
    const int n = g.t1 - g.t0;
    if (g.solo == 1) {
      couple = ring;
      ring += 2 * (n + g.other);
    }
    if (g.solo && g.solo - 1 != w) continue;
    const bool pair = g.nrows > p.tile_rows, alone = pair || g.solo;  // alone: a row tile is this stream's only
    const int steps = alone ? n : (n + 1 - w) / 2;
    const int rl = (pair ? w * p.tile_rows : 0) + tid;  // this thread's row of the item
    const bool inside = tid < p.tile_rows && rl < g.nrows;
    const int r = g.r0 + rl, node = inside ? r / p.group : 0;
    const int* const table = p.c.table + static_cast<long long>(max(g.row, 0)) * p.c.max_pages;
    if (g.first != had_first || g.row != had_row || g.r0 != had_r0) {  // other heads of the same rows see the same
      had_first = g.first;
      had_row = g.row;
      had_r0 = g.r0;
      see.tree = p.parents != nullptr;
      see.len = g.len;
      see.upto = g.len + node + 1;
      see.used = inside && g.row >= 0;
      if (see.tree) {
        short* const up = sh->row[w].up;
        const int nodes = g.row < 0 ? 0 : g.nodes;
        for (int j = tid; j < nodes; j += kRows) {
          const int u = p.parents[g.first + j];
          const bool odd = u < -2 || u >= j;
          if (odd) atomicOr(p.status, kStatusBadSeq);
          up[j] = static_cast<short>(odd ? -2 : u);
        }
        named_bar_sync(1 + w, kRows);
        see.used = see.used && up[node] >= -1;
        int j = see.used ? node : -1;
#pragma unroll
        for (int i = kTreeMaxNodes / 32 - 1; i >= 0; --i) {  // parents come before their children
          unsigned on = 0u;
          while (j >= 32 * i) {
            const int above = up[j];
            if (above >= -1) on |= 1u << (j & 31);
            j = above;
          }
          see.path[i] = on;
        }
        named_bar_sync(1 + w, kRows);
      }
    }
    const bool busy = __any_sync(0xffffffffu, inside);  // rows of this warp
    float m = -INFINITY, l = 0.f;
    for (int i = 0; i < steps; ++i) {
      const int j = alone ? i : 2 * i + w, k0 = (g.t0 + j) * kKeys;
      const bool masked = k0 + kKeys > g.all;
      // (Before anything else: that S is there says that what the ring held before this step's V has arrived, without
      // which a wait for V, by parity, could take an earlier round's arrival for it.)
      wait(p, sh, &sh->s_full[w], s_par);
      s_par ^= 1u;
      tc_fence_after();
      if (masked) {
        // Values that not every row sees: infinities and NaN become 0, to be added to the rows that see them at
        // the end.  Those behind the last key, up to the end of its page, become 0 (the pages behind it came as
        // zeros).  Where the other stream has the same tile, one of the two finds what there is: it says so before
        // it clears anything, and the other, which looks at `fix` when both are through, has seen either.
        const int n0 = g.solo == 2 ? g.other : g.solo ? n : (n + 1) / 2, n1 = g.solo == 1 ? g.other : g.solo ? n : n / 2;
        const uint32_t at = pair ? ring + 2 * i + 1 : (g.solo ? couple : ring) + place_v(n0, n1, w, i), stage = at % L::kStages;
        const uint32_t tile = base + L::kRing + stage * L::kTile;
        const int a = max(g.all - k0, 0), b = min((g.total + mask & ~mask) - k0, kKeys), last = g.total - k0;
        wait(p, sh, &sh->full[stage], (at / L::kStages) & 1u);
#pragma unroll 4
        for (int x = a * DC * 8 + tid; x < b * DC * 8; x += kRows) {
          const int row = x / (DC * 8), c = x % (DC * 8);
          const uint32_t addr = tile + L::at(row, c);
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (row < last) {
            v = ld_shared_v4(addr);
            if (!odd_any(v)) continue;
            *static_cast<volatile int*>(&sh->fix[seg & 3]) = seg;
            __threadfence_block();
            uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              if (odd_lo(u[y])) u[y] &= 0xffff0000u;
              if (odd_hi(u[y])) u[y] &= 0x0000ffffu;
            }
            v = make_uint4(u[0], u[1], u[2], u[3]);
          }
          st_shared_v4(addr, v.x, v.y, v.z, v.w);
        }
        fence_proxy_async_smem();
        __threadfence_block();
      }
      if (busy) {
        float z[kKeys];
        tmem_ld128(ts, z);
        if (masked) {
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const unsigned b = see.bits(k0 + 32 * x);
#pragma unroll
            for (int y = 0; y < 32; ++y) z[32 * x + y] = (b >> y) & 1u ? z[32 * x + y] : -INFINITY;
          }
        }
        float top[4] = {z[0], z[1], z[2], z[3]};
#pragma unroll
        for (int x = 4; x + 8 <= kKeys; x += 8)
#pragma unroll
          for (int y = 0; y < 4; ++y) top[y] = fmax3(top[y], z[x + y], z[x + 4 + y]);
        const float now = fmax3(fmaxf(top[0], z[kKeys - 4]), fmax3(top[1], z[kKeys - 3], top[2]),
                                fmax3(top[3], z[kKeys - 2], z[kKeys - 1]));
        // The maximum moves only where it must; where it does, what is summed so far is brought down.
        const bool move = (now - m) * p.scale > kGrow || (m == -INFINITY && now > m);
        if (__any_sync(0xffffffffu, move)) {
          const float c = !move ? 1.f : m == -INFINITY ? 0.f : fast_exp2(tree_base(p, m) - tree_base(p, now));
          if (move) m = now;
          l *= c;
          if (i > 0) {
#pragma unroll 1
            for (int x = 0; x < p.dim; x += 32) {
              float o[32];
              tmem_ld32(to + x, o);
              uint32_t u[32];
#pragma unroll
              for (int y = 0; y < 32; ++y) u[y] = __float_as_uint(o[y] * c);
              tmem_st32(to + x, u);
            }
          }
        }
        const float off = -tree_base(p, m);
        const float2 scale2 = make_float2(p.scale, p.scale), off2 = make_float2(off, off);
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        // The MMAs of the first half of the keys begin while the second half's exponentials are taken.
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t u[kKeys / 4];
#pragma unroll
          for (int x = 0; x < kKeys / 2; x += 2) {
            const float2 e = fma2(make_float2(z[64 * h + x], z[64 * h + x + 1]), scale2, off2);
            const float2 f = make_float2(fast_exp2(e.x), fast_exp2(e.y));
            sum[(x >> 1) & 1] = add2(sum[(x >> 1) & 1], f);
            u[x / 2] = pack_bf16(f.x, f.y);
          }
          tmem_st32(ts + 32 * h, u);
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&sh->p_ready[w][h]));
        }
        l += (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
      } else {
        __syncwarp();
        if (lane == 0)
          for (int h = 0; h < 2; ++h) mbar_arrive(smem_u32(&sh->p_ready[w][h]));
      }
    }
    if (!g.solo) ring += 2 * n;

    // The end of a segment.  Streams of one row tile meet here: both read both accumulators, half of the columns
    // each, which is why neither goes on before the other has read.
    if (steps > 0) {
      wait(p, sh, &sh->o_full[w], o_par);
      o_par ^= 1u;
    }
    float c_own = 1.f, c_other = 0.f, M = m, Lsum = l;
    if (!alone) {
      sh->row[w].ml[tid] = make_float2(m, l);
      tc_fence_before();
      meet();
      const float2 o = sh->row[1 - w].ml[tid];
      M = fmaxf(m, o.x);
      const float off = tree_base(p, M);
      c_own = l == 0.f ? 0.f : m == -INFINITY ? 1.f : fast_exp2(tree_base(p, m) - off);
      c_other = o.y == 0.f ? 0.f : o.x == -INFINITY ? 1.f : fast_exp2(tree_base(p, o.x) - off);
      // (A sum without a maximum is NaN and stays so.)
      Lsum = (l == 0.f ? 0.f : l * c_own) + (o.y == 0.f ? 0.f : o.y * c_other);
    }
    tc_fence_after();
    const bool fix = *static_cast<volatile int*>(&sh->fix[seg & 3]) == seg;
    const bool whole = g.t0 == 0 && g.t1 == g.nt;
    const float inv = whole ? (Lsum == 0.f || !see.used ? 0.f : 1.f / Lsum) : 1.f;
    const int chunks = (p.dim + 31) / 32;
    const int x0 = alone || w == 0 ? 0 : (chunks + 1) / 2, x1 = alone || w == 1 ? chunks : (chunks + 1) / 2;
    const int out_row = tree_out_row(p, g.first, g.head, inside ? r : g.r0);
    // A piece's rows lie side by side, four values each, so that the lanes' stores do.
    const int rows = p.part_rows;
    float* const part = tree_part(p, blockIdx.x, g.slot);
    const uint32_t other = tmem + lanes + kAccO + (1 - w) * 128;
    if (busy) {
      // For stores of 64 bytes of a row, four lanes exchange their 16 bytes of each other's rows.
      const int four = lane & 3;
      int row4[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) row4[y] = __shfl_sync(0xffffffffu, inside ? out_row : -1, (lane & ~3) + y);
#pragma unroll 1
      for (int x = x0; x < x1; ++x) {
        float o[32];
#pragma unroll
        for (int y = 0; y < 32; ++y) o[y] = 0.f;
        if (steps > 0) {
          float v[32];
          tmem_ld32(to + 32 * x, v);
#pragma unroll
          for (int y = 0; y < 32; ++y) o[y] = c_own == 0.f ? 0.f : v[y] * c_own;
        }
        if (!alone && n > 1 - w) {                  // the other stream had a tile too
          float v[32];
          tmem_ld32(other + 32 * x, v);
#pragma unroll
          for (int y = 0; y < 32; ++y) o[y] += c_other == 0.f ? 0.f : v[y] * c_other;
        }
        if (fix) {
          const int b = min(g.total, g.t1 * kKeys);
          for (int k = max(g.all, g.t0 * kKeys); k < b; ++k) {
            const int page = table[k >> p.c.page_shift];
            if (!(see.bits(k) & 1u) || page < 0 || page >= p.c.pages) continue;
            const __nv_bfloat16* const v = V + cache_at(p.c, p.layer, page, g.head, k & mask) * 8 + 32 * x;
#pragma unroll
            for (int y = 0; y < 32; ++y)
              if (32 * x + y < p.dim) {
                const float f = __bfloat162float(v[y]);
                if (!isfinite(f)) o[y] += f;
              }
          }
        }
        __syncwarp();
        if (whole) {
          uint32_t u[4][4];
#pragma unroll
          for (int y = 0; y < 16; ++y)
            u[y >> 2][y & 3] = see.used ? pack_bf16(o[2 * y] * inv, o[2 * y + 1] * inv) : 0u;
#pragma unroll
          for (int d = 1; d < 4; d <<= 1)
#pragma unroll
            for (int a = 0; a < 4; ++a)
              if (!(a & d))
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                  const bool up = four & d;
                  const uint32_t give = __shfl_xor_sync(0xffffffffu, up ? u[a][y] : u[a + d][y], d);
                  if (up) u[a][y] = give;
                  else u[a + d][y] = give;
                }
          __nv_bfloat16* const out = static_cast<__nv_bfloat16*>(p.out) + 32 * x + 8 * four;
#pragma unroll
          for (int y = 0; y < 4; ++y)
            if (row4[y] >= 0 && 32 * x + 8 * four < p.dim)
              st16(out + static_cast<long long>(row4[y]) * p.dim, make_uint4(u[y][0], u[y][1], u[y][2], u[y][3]));
        } else if (inside) {
          float4* const at = reinterpret_cast<float4*>(part + 4 * rows) + static_cast<long long>(8 * x) * rows + rl;
#pragma unroll
          for (int y = 0; y < 8; ++y)
            if (32 * x + 4 * y < p.dim) at[y * rows] = make_float4(o[4 * y], o[4 * y + 1], o[4 * y + 2], o[4 * y + 3]);
        }
      }
    }
    if (inside && (alone || w == 0)) {
      const float sum = see.used ? Lsum : 0.f;
      if (whole) p.lse[out_row] = tree_lse(p, M, sum);
      else reinterpret_cast<float2*>(part)[rl] = make_float2(M, sum);
    }
    tc_fence_before();
    if (!alone) meet();
  }
}

template <int DC, bool kJoint>
__global__ void __launch_bounds__(kThreads, 1) tree_kernel(const __grid_constant__ TreeParams p) {
  using L = Layout<DC, kJoint>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t base = smem_u32(smem);
  Tail* const sh = reinterpret_cast<Tail*>(smem + L::kTail);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    plan_init(sh, kSegReaders);
    for (int& f : sh->fix) f = 0;
    for (int s = 0; s < L::kStages; ++s) {
      mbar_init(smem_u32(&sh->full[s]), 1);
      mbar_init(smem_u32(&sh->empty[s]), 1);
    }
    for (int w = 0; w < 2; ++w) {
      mbar_init(smem_u32(&sh->q_ready[w]), 1);
      mbar_init(smem_u32(&sh->q_free[w]), 1);
      mbar_init(smem_u32(&sh->s_full[w]), 1);
      for (int h = 0; h < 2; ++h) mbar_init(smem_u32(&sh->p_ready[w][h]), kRows / 32);
      mbar_init(smem_u32(&sh->o_full[w]), 1);
    }
    mbar_init(smem_u32(&sh->met), 8);
    mbar_init(smem_u32(&sh->drain), 1);
    fence_barrier_init();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&sh->tmem_slot), kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  const Range range = plan_cut<kThreads>(p, sh);  // has barriers
  tc_fence_after();
  const uint32_t tmem = sh->tmem_slot;
  chain_trigger();  // every CTA of this launch is resident: the next kernel's cannot take their place

  if (warp < 4) {
    regs_decrease<kCtlRegs>();
    if (warp == 0) {
      load_role<DC, kJoint>(p, sh, base);
    } else if (warp == 1) {
      mma_role<DC, kJoint>(p, sh, base, tmem);
    } else if (warp == 2) {
      if (lane == 0) plan_role(p, sh, range);
    } else {
      query_role<DC>(p, sh, base);
    }
    __syncwarp();
  } else {
    regs_increase<kSoftmaxRegs>();
    softmax_role<DC, kJoint>(p, sh, base, tmem, (warp - 4) >> 2);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

}  // namespace

// Rows of a tile: whole nodes, as many as it holds, or any of a larger group.
int tree_tile_rows(int group) { return group <= kRows ? kRows / group * group : kRows; }
// Rows of a box of queries (0: none takes them): where tiles are full, as few nodes as make whole atoms of 8 rows,
// so that few nodes bring few; else the tile's, as boxes have to begin with an atom.
int tree_query_rows(int group) {
  return group > kRows ? 0 : kRows % group ? kRows / group * group : group < 8 ? 8 : group;
}

cudaError_t launch_tree_bf16(const TreeParams& p, cudaStream_t s) {
  const int grid = p.sms;
  if (p.joint) tree_kernel<2, true><<<grid, kThreads, kSmem, s>>>(p);
  else if (p.dim > 64) tree_kernel<2, false><<<grid, kThreads, kSmem, s>>>(p);
  else tree_kernel<1, false><<<grid, kThreads, kSmem, s>>>(p);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  return launch_tree_join(p, s);
}

cudaError_t setup_tree_mma_kernels() {
  for (void (*kernel)(TreeParams) : {tree_kernel<1, false>, tree_kernel<2, false>, tree_kernel<2, true>}) {
    cudaFuncAttributes fa;
    cudaError_t e = cudaFuncGetAttributes(&fa, kernel);
    if (e != cudaSuccess) return e;
    // The split of registers between the roles waits forever unless the launch has just that many.
    if (fa.numRegs != kLaunchRegs || fa.maxThreadsPerBlock < kThreads) return cudaErrorInvalidConfiguration;
    if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem)) != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace mls
