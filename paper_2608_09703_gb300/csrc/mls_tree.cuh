// What the tree-attention kernels share: the entries of a call.
#pragma once

#include "mls_device.cuh"
#include "mls_kernels.h"

namespace mls {

constexpr float kLn2 = 0.6931471805599453f;

// What an entry of a call is: its nodes [first, first + nodes) of the packed ones, its row of the
// table and the tokens cached there.  What does not fit the cache is an entry of unused nodes.
struct Entry {
  int nodes, row, len;
  long long first;
};
__device__ __forceinline__ Entry tree_entry(const TreeParams& p, int i, int* status) {
  Entry e;
  const long long a = p.start[i], b = p.start[i + 1];
  bool bad = a < 0 || b < a || b > p.N;
  e.first = a;
  e.nodes = bad ? 0 : static_cast<int>(b - a);
  e.row = p.seqs ? p.seqs[i] : i;
  e.len = 0;
  if (e.nodes) {
    if (e.row < 0 || e.row >= p.c.seqs || (p.parents && e.nodes > kTreeMaxNodes)) {
      bad = true;
      e.row = -1;
    } else {
      e.len = p.c.len[e.row];
      if (e.len < 0 || static_cast<long long>(e.len) + e.nodes > (static_cast<long long>(p.c.max_pages) << p.c.page_shift)) {
        bad = true;
        e.row = -1;
        e.len = 0;
      }
    }
  }
  if (bad) atomicOr(status, kStatusBadSeq);
  return e;
}

}  // namespace mls
