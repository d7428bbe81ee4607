// The pages of a key/value cache: taking, sharing, filling, closing up and giving back.
//
// A page is free exactly while its count of references is 0, and the free pages are also
// a bit each in free_bits.  Pages are always taken from the lowest-numbered free one on, in
// the order of a call's entries.  So where everything lies follows from the calls alone: counts
// change by integer atomics whose order does not matter, and no list remembers an order.
//
// What moves data (append, fork, compact, copy) reads each byte once and writes it once, in
// pieces of 16 bytes, several of them in flight per thread; HBM bounds it.  (Not where an append has
// thousands of entries: each of its blocks looks at all offsets, and 8192 of a token each take 68 us
// where their bytes take 10.)  The rest touches a few words per page and is bound by the latency of
// its chain of loads.
//
// The calls take entries (rows of the table) in strictly increasing order, which every
// block can check for its own entry by looking at those before it.
#include <climits>

#include "mls_device.cuh"
#include "mls_kernels.h"

namespace mls {
namespace {

constexpr int kThreads = 256;
constexpr int kTake = 1024;  // threads of the kernel that hands out pages

__device__ __forceinline__ bool page_ok(const CacheView& c, int page) { return page >= 0 && page < c.pages; }
__device__ __forceinline__ int clamp_held(const CacheView& c, int row) { return min(max(c.held[row], 0), c.max_pages); }

// The table row of entry i, or -1 if it is not greater than all before it or not one of the
// cache's.  The whole block calls it.
__device__ int entry_row(const CacheView& c, const int* seqs, int i) {
  if (!seqs) return i;
  const int id = seqs[i];
  int bad = id < 0 || id >= c.seqs;
  for (int j = threadIdx.x; j < i; j += blockDim.x) bad |= seqs[j] >= id;
  bad = __syncthreads_or(bad);
  if (bad && threadIdx.x == 0) atomicOr(c.status, kStatusBadSeq);
  return bad ? -1 : id;
}

// One reference less for the pages in columns [from, to) of a row, whose places become -1.
__device__ void drop_pages(const CacheView& c, int row, int from, int to) {
  for (int col = from + threadIdx.x; col < to; col += blockDim.x) {
    int* const at = c.table + static_cast<long long>(row) * c.max_pages + col;
    const int page = *at;
    *at = -1;
    if (!page_ok(c, page)) {
      atomicOr(c.status, kStatusBadSeq);
      continue;
    }
    const int old = atomicSub(c.refs + page, 1);
    if (old == 1) {
      atomicOr(c.free_bits + (page >> 5), 1u << (page & 31));
    } else if (old < 1) {  // it was free already: the table does not fit the counts
      atomicAdd(c.refs + page, 1);
      atomicOr(c.status, kStatusBadSeq);
    }
  }
}

__global__ void reset_kernel(CacheView c) {
  const long long t = static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x;
  const long long step = static_cast<long long>(gridDim.x) * blockDim.x;
  for (long long i = t; i < static_cast<long long>(c.seqs) * c.max_pages; i += step) c.table[i] = -1;
  for (long long i = t; i < c.seqs; i += step) c.len[i] = c.held[i] = 0;
  for (long long i = t; i < c.pages; i += step) c.refs[i] = 0;
  for (long long i = t; i * 32 < c.pages; i += step) {
    const long long left = c.pages - i * 32;
    c.free_bits[i] = left >= 32 ? 0xffffffffu : (1u << left) - 1u;
  }
}

__global__ void __launch_bounds__(kThreads) free_kernel(CacheView c, const int* seqs) {
  const int row = entry_row(c, seqs, blockIdx.x);
  if (row < 0) return;
  const int held = clamp_held(c, row);
  drop_pages(c, row, 0, held);
  __syncthreads();  // every thread has read held
  if (threadIdx.x == 0) c.len[row] = c.held[row] = 0;
}

// Sums over the threads before this one and over all, of a block of kTake threads.
__device__ void block_scan(int v, int& before, int& all) {
  __shared__ int warp_sums[kTake / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int upto = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int w = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += w;
  }
  if (lane == 31) warp_sums[warp] = upto;
  __syncthreads();
  int s = warp_sums[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int w = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += w;
  }
  const int warps_before = __shfl_sync(0xffffffffu, s, (warp + 31) & 31);
  before = upto - v + (warp ? warps_before : 0);
  all = __shfl_sync(0xffffffffu, s, 31);
  __syncthreads();  // before the sums are written again
}

// Largest value among the threads before this one, and among all (-1 if there are none).
__device__ void block_max_before(int v, int& before, int& all) {
  __shared__ int warp_max[kTake / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int upto = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int w = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto = max(upto, w);
  }
  if (lane == 31) warp_max[warp] = upto;
  int prev = __shfl_up_sync(0xffffffffu, upto, 1);
  if (lane == 0) prev = -1;
  __syncthreads();
  int m = warp_max[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int w = __shfl_up_sync(0xffffffffu, m, o);
    if (lane >= o) m = max(m, w);
  }
  const int warps_before = __shfl_sync(0xffffffffu, m, (warp + 31) & 31);
  before = warp ? max(prev, warps_before) : prev;
  all = __shfl_sync(0xffffffffu, m, 31);
  __syncthreads();
}

// Hands out pages to the entries of a reserve (as many as it takes to hold len + count tokens)
// or of a fork (one, where the source's last page is partly filled).  One block: the entries' needs
// become a prefix in shared memory, the free pages of the bit map are ranked by their count of
// bits, and the page of rank r goes to the entry whose range of the prefix holds r.  A warp takes a word of
// the map at a time, a lane a page (a thread a word: 12.5 us for 64 entries and some 3500 pages, so 6.3).
template <bool kFork>
__global__ void __launch_bounds__(kTake)
    take_kernel(CacheView c, int n, const int* seqs, const int* count, const int* src, int* fresh, int* length) {
  extern __shared__ int pre[];  // [n + 1]
  __shared__ unsigned s_bits[kTake];
  __shared__ int s_rank[kTake];
  const int tid = threadIdx.x, lane = tid & 31;
  const int words = (c.pages + 31) >> 5;
  const unsigned first_bits = tid < words ? c.free_bits[tid] : 0u;  // on its way while the entries are looked at
  int total = 0, top = -1;
  bool wide = false;
  for (int i0 = 0; i0 < n; i0 += kTake) {
    const int i = i0 + tid;
    const int id = i < n ? (seqs ? seqs[i] : i) : -1;
    int before, all;
    block_max_before(id, before, all);
    int need = 0;
    if (i < n) {
      const bool ok = id >= 0 && id < c.seqs && id > max(before, top);
      int bits = ok ? 0 : kStatusBadSeq;
      const long long size = 1LL << c.page_shift;
      if constexpr (kFork) {
        const int from = src[i];
        int f = -2, len = 0;
        if (ok) {
          if (from < 0 || from >= c.seqs || c.held[id] != 0) {
            bits = kStatusBadSeq;
          } else {
            len = max(c.len[from], 0);
            const int pages = static_cast<int>((len + size - 1) >> c.page_shift);
            if (pages > clamp_held(c, from)) {
              bits = kStatusBadSeq;
            } else {
              f = -1;
              need = (len & (size - 1)) != 0;
            }
          }
        }
        fresh[i] = f;
        length[i] = len;
      } else if (ok) {
        const int more = count[i];
        const int have = clamp_held(c, id);
        if (more < 0) {
          bits = kStatusBadSeq;
        } else {
          const long long pages = (max(c.len[id], 0) + static_cast<long long>(more) + size - 1) >> c.page_shift;
          if (pages > c.max_pages) bits = kStatusNoPages;
          else need = static_cast<int>(max(pages - have, 0LL));
        }
      }
      if (bits) atomicOr(c.status, bits);
    }
    top = max(top, all);
    // A row has at most 2^20 pages and a cache 2^26, so a turn's sum and `total` stay within 32
    // bits; once more is asked for than there are pages, no later entry is served.
    int b, a;
    block_scan(need, b, a);
    if (i < n) pre[i] = wide ? INT_MAX : total + b;
    if (!wide) total += a;
    wide = total > c.pages;
  }
  if (tid == 0) pre[n] = wide ? INT_MAX : total;
  int mine = __popc(first_bits);
  for (int w = tid + kTake; w < words; w += kTake) mine += __popc(c.free_bits[w]);
  int skip, avail;
  block_scan(mine, skip, avail);  // also orders pre[] before its readers
  // Entries are served while their pages and those of all before them are there.
  int lo = 0, hi = n;             // the first entry that is not: pre[lo + 1] > avail
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid + 1] > avail) hi = mid;
    else lo = mid + 1;
  }
  const int served = lo, limit = pre[served];
  if (served < n && tid == 0) atomicOr(c.status, kStatusNoPages);
  int given = 0;
  for (int w0 = 0; w0 < words && given < limit; w0 += kTake) {
    const int w = w0 + tid;
    const unsigned bits = w0 == 0 ? first_bits : w < words ? c.free_bits[w] : 0u;
    int before = skip, all = avail;
    if (words > kTake) block_scan(__popc(bits), before, all);
    s_bits[tid] = bits;
    s_rank[tid] = given + before;
    given += all;
    __syncthreads();
    for (int x = tid >> 5; x < kTake && w0 + x < words && s_rank[x] < limit; x += kTake / 32) {
      const unsigned b = s_bits[x];
      const int r = s_rank[x] + __popc(b & ((1u << lane) - 1u));
      const bool mine_too = (b >> lane & 1u) && r < limit;
      if (mine_too) {
        const int page = (w0 + x) * 32 + lane;
        MLS_CHECK(c.status, page < c.pages && c.refs[page] == 0);
        int e = 0, e1 = served - 1;  // the last entry whose range begins at or before r: it is not empty
        while (e < e1) {
          const int mid = (e + e1 + 1) >> 1;
          if (pre[mid] <= r) e = mid;
          else e1 = mid - 1;
        }
        if constexpr (kFork) {
          fresh[e] = page;
        } else {
          const int row = seqs ? seqs[e] : e;
          MLS_CHECK(c.status, e < served && r >= pre[e] && r < pre[e + 1] && clamp_held(c, row) + (r - pre[e]) < c.max_pages);
          c.table[static_cast<long long>(row) * c.max_pages + clamp_held(c, row) + (r - pre[e])] = page;
        }
        c.refs[page] = 1;
      }
      const unsigned gone = __ballot_sync(0xffffffffu, mine_too);
      if (lane == 0 && gone) c.free_bits[w0 + x] = b & ~gone;
    }
    __syncthreads();
  }
  __syncthreads();
  for (int i = tid; i < n; i += kTake) {
    if constexpr (kFork) {
      if (i >= served && fresh[i] == -1 && (length[i] & ((1 << c.page_shift) - 1))) fresh[i] = -2;
    } else if (i < served && pre[i + 1] > pre[i]) {
      const int row = seqs ? seqs[i] : i;
      c.held[row] = clamp_held(c, row) + pre[i + 1] - pre[i];
    }
  }
}

// Copies the first `slots` tokens of a page to another, for all layers and heads, spread over
// gridDim.y blocks.  kDeep copies of 16 bytes are in flight per thread.
constexpr int kDeep = 8;
__device__ void copy_page(const CacheView& from, const CacheView& to, int src, int dst, int slots) {
  // Pieces of a head lie side by side; all of a page's are counted in 32 bits.  (In 64, whose division is slow, forking
  // 64 prompts of 28 layers took 26 us, so 23.)
  const unsigned each = static_cast<unsigned>(slots) * from.row, planes = 2u * from.layers * from.heads;
  const unsigned all = each * planes, step = gridDim.y * blockDim.x;
  MLS_CHECK(from.status, page_ok(from, src) && page_ok(to, dst) && slots <= 1 << from.page_shift);
  for (unsigned i = blockIdx.y * blockDim.x + threadIdx.x; i < all; i += step * kDeep) {
    uint4 v[kDeep];
    uint4* at[kDeep];
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
      const unsigned x = i + j * step;
      at[j] = nullptr;
      if (x >= all) continue;
      const unsigned plane = x / each, piece = x - plane * each, lk = plane / from.heads;
      const int head = static_cast<int>(plane - lk * from.heads), layer = static_cast<int>(lk >> 1);
      v[j] = ((lk & 1) ? from.v : from.k)[cache_at(from, layer, src, head, 0) + piece];
      at[j] = ((lk & 1) ? to.v : to.k) + cache_at(to, layer, dst, head, 0) + piece;
    }
#pragma unroll
    for (int j = 0; j < kDeep; ++j)
      if (at[j]) *at[j] = v[j];
  }
}

__global__ void __launch_bounds__(kThreads)
    fork_kernel(CacheView c, const int* src, const int* dst, const int* fresh, const int* length) {
  chain_wait();
  const int i = blockIdx.x, f = fresh[i];
  if (f == -2) return;
  const int from = src[i], to = dst ? dst[i] : i, len = length[i];
  const int full = len >> c.page_shift, part = len & ((1 << c.page_shift) - 1);
  const int* const row = c.table + static_cast<long long>(from) * c.max_pages;
  if (blockIdx.y > 0 && part == 0) return;
  const int last = part ? row[full] : 0;
  // A source with a page that is none is left out, and the page taken for the copy is free again.  Each block
  // looks, so that none writes: 0.6 of 14.3 us for 64 samples of 28 layers.
  int bad = !page_ok(c, last);
  for (int col = threadIdx.x; col < full; col += blockDim.x) bad |= !page_ok(c, row[col]);
  if (__syncthreads_or(bad)) {
    if (blockIdx.y == 0 && threadIdx.x == 0) {
      atomicOr(c.status, kStatusBadSeq);
      if (part) {
        c.refs[f] = 0;
        atomicOr(c.free_bits + (f >> 5), 1u << (f & 31));
      }
    }
    return;
  }
  if (blockIdx.y == 0) {
    int* const out = c.table + static_cast<long long>(to) * c.max_pages;
    for (int col = threadIdx.x; col < full; col += blockDim.x) {
      const int page = row[col];
      out[col] = page;
      atomicAdd(c.refs + page, 1);
    }
    if (threadIdx.x == 0) {
      if (part) out[full] = f;
      c.held[to] = full + (part != 0);
      c.len[to] = len;
    }
  }
  if (part) copy_page(c, c, last, f, part);
}

__global__ void __launch_bounds__(kThreads) copy_kernel(CacheView from, CacheView to, const int* src, const int* dst) {
  const int a = src[blockIdx.x], b = dst[blockIdx.x];
  if (!page_ok(from, a) || !page_ok(to, b)) {
    if (threadIdx.x == 0) atomicOr(from.status, kStatusBadSeq);
    return;
  }
  copy_page(from, to, a, b, 1 << from.page_shift);
}

// A block writes one token (gridDim.y of them share its layers).
__global__ void __launch_bounds__(kThreads) append_kernel(CacheView c, CacheAppend a) {
  __shared__ int entry;
  const long long t = blockIdx.x;
  if (threadIdx.x == 0) entry = INT_MAX;
  __syncthreads();
  // Each block looks at all offsets.  Of the entries whose own are in order only the first that holds the token can
  // have it: one behind it that holds it too begins before the end of the first, where the entry after the first begins.
  int bad = 0;
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    const int from = a.start[i], to = a.start[i + 1];
    if (from < 0 || to < from || to > a.N) bad = 1;
    else if (from <= t && t < to) atomicMin(&entry, i);
  }
  bad = __syncthreads_or(bad);
  const int i = entry;
  if (bad) {
    if (threadIdx.x == 0) atomicOr(c.status, kStatusBadSeq);
    int late = 0;  // it begins before one in front of it does
    for (int j = threadIdx.x; i < a.n && j < i; j += blockDim.x) late |= a.start[j] > a.start[i];
    if (__syncthreads_or(late)) return;
  }
  if (i >= a.n) return;  // a token of no entry
  const int row = entry_row(c, a.seqs, i);
  if (row < 0) return;
  const long long at = c.len[row] + (t - a.start[i]);
  const long long col = at >> c.page_shift;
  const int page = at >= 0 && col < clamp_held(c, row) ? c.table[static_cast<long long>(row) * c.max_pages + col] : -1;
  if (!page_ok(c, page)) {
    if (threadIdx.x == 0) atomicOr(c.status, kStatusNoPages);
    return;
  }
  const int slot = static_cast<int>(at & ((1 << c.page_shift) - 1));
  MLS_CHECK(c.status, t >= a.start[i] && t < a.start[i + 1] && t < a.N && a.layer0 + a.layers <= c.layers);
  const int each = c.heads * c.row, all = 2 * a.layers * each;
  const int step = gridDim.y * blockDim.x;
  constexpr int kAhead = 4;
  for (int x0 = blockIdx.y * blockDim.x + threadIdx.x; x0 < all; x0 += step * kAhead) {
    uint4 v[kAhead];
    uint4* out[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const long long x = x0 + static_cast<long long>(j) * step;
      out[j] = nullptr;
      if (x >= all) continue;
      const int lk = static_cast<int>(x) / each, piece = static_cast<int>(x) - lk * each, layer = lk >> 1;
      const int head = piece / c.row;
      v[j] = ((lk & 1) ? a.v : a.k)[layer * a.layer_ld + t * a.token_ld + piece];
      out[j] = ((lk & 1) ? c.v : c.k) + cache_at(c, a.layer0 + layer, page, head, slot) + (piece - head * c.row);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (out[j]) *out[j] = v[j];
  }
}

// Whether an entry's path may be kept: 0 <= path[0] < path[1] < ... < what is there behind its
// len tokens, in pages that are all the cache's.  Then path[k] >= k.  Also the first k with path[k] != k.
// The whole block calls it; all of an entry's blocks find the same, as nothing here changes before its closing.
__device__ bool path_ok(const CacheView& c, int row, const int* path, int path_ld, int keep, int len, int held,
                        int& first) {
  const long long room = (static_cast<long long>(held) << c.page_shift) - len;
  int bad = keep < 0 || keep > room || len < 0 || (path && keep > path_ld);
  int moved = 0;
  if (!bad)
    for (int col = (len >> c.page_shift) + threadIdx.x; col < held; col += blockDim.x)
      bad |= !page_ok(c, c.table[static_cast<long long>(row) * c.max_pages + col]);
  if (path && !bad)
    for (int k = threadIdx.x; k < keep; k += blockDim.x) {
      const int at = path[k];
      bad |= at < 0 || at >= room || (k > 0 && path[k - 1] >= at);
      moved |= at != k;
    }
  bad = __syncthreads_or(bad);
  first = keep;
  if (bad || !path || !__syncthreads_or(moved)) return !bad;
  __shared__ int low;
  if (threadIdx.x == 0) low = keep;
  __syncthreads();
  for (int k = threadIdx.x; k < keep; k += blockDim.x)
    if (path[k] != k) {
      atomicMin(&low, k);
      break;
    }
  __syncthreads();
  first = low;
  return true;
}

// The lengths that are kept, and the pages behind them given back.
__device__ void close_entry(const CacheView& c, int row, int n, int len, int held) {
  const int pages = (len + n + (1 << c.page_shift) - 1) >> c.page_shift;
  drop_pages(c, row, pages, held);
  __syncthreads();  // every thread has read len and held
  if (threadIdx.x == 0) {
    c.len[row] = len + n;
    c.held[row] = pages;
  }
}

// Moves the kept tokens of an entry together.  A thread has one piece of 16 bytes of a head and
// layer and walks the path: since path[k] >= k and the path increases, what it writes at k lies
// before all that it has still to read, so the move is right in place, several tokens at a time.
// An entry's only block closes it too (kClose).
template <bool kClose>
__global__ void __launch_bounds__(kThreads)
    move_kernel(CacheView c, const int* seqs, const int* keep, const int* path, int path_ld) {
  __shared__ int src_page[kCachePath], dst_page[kCachePath];
  __shared__ short src_slot[kCachePath], dst_slot[kCachePath];
  const int row = entry_row(c, seqs, blockIdx.x);
  if (row < 0) return;
  const int* const mine = path + static_cast<long long>(blockIdx.x) * path_ld;
  const int n = keep[blockIdx.x], len = c.len[row], held = clamp_held(c, row);
  int first;
  if (!path_ok(c, row, mine, path_ld, n, len, held, first)) {
    if (kClose && threadIdx.x == 0) atomicOr(c.status, kStatusBadSeq);  // else the next kernel says so
    return;
  }
  const int* const table = c.table + static_cast<long long>(row) * c.max_pages;
  const int mask = (1 << c.page_shift) - 1;
  const int pieces = 2 * c.layers * c.heads * c.row;
  for (int k0 = first; k0 < n; k0 += kCachePath) {
    const int m = min(kCachePath, n - k0);
    __syncthreads();
    for (int k = threadIdx.x; k < m; k += blockDim.x) {
      const long long a = static_cast<long long>(len) + mine[k0 + k], b = static_cast<long long>(len) + k0 + k;
      src_page[k] = table[a >> c.page_shift];
      dst_page[k] = table[b >> c.page_shift];
      src_slot[k] = static_cast<short>(a & mask);
      dst_slot[k] = static_cast<short>(b & mask);
      MLS_CHECK(c.status, b <= a && (a >> c.page_shift) < held && page_ok(c, src_page[k]) && page_ok(c, dst_page[k]));
    }
    __syncthreads();
    for (int x = blockIdx.y * blockDim.x + threadIdx.x; x < pieces; x += gridDim.y * blockDim.x) {
      const int piece = x % c.row, plane = x / c.row, head = plane % c.heads, lk = plane / c.heads;
      uint4* const pool = ((lk & 1) ? c.v : c.k) + piece;
      constexpr int kAhead = 8;
      for (int k = 0; k < m; k += kAhead) {
        uint4 v[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
          if (k + j < m) v[j] = pool[cache_at(c, lk >> 1, src_page[k + j], head, src_slot[k + j])];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
          if (k + j < m) pool[cache_at(c, lk >> 1, dst_page[k + j], head, dst_slot[k + j])] = v[j];
      }
    }
  }
  if (kClose) {
    __syncthreads();  // the table is read until here
    close_entry(c, row, n, len, held);
  }
}

__global__ void __launch_bounds__(kThreads)
    close_kernel(CacheView c, const int* seqs, const int* keep, const int* path, int path_ld) {
  chain_wait();
  const int row = entry_row(c, seqs, blockIdx.x);
  if (row < 0) return;
  const int* const mine = path ? path + static_cast<long long>(blockIdx.x) * path_ld : nullptr;
  const int n = keep[blockIdx.x], len = c.len[row], held = clamp_held(c, row);
  int first;
  if (!path_ok(c, row, mine, path_ld, n, len, held, first)) {
    if (threadIdx.x == 0) atomicOr(c.status, kStatusBadSeq);
    return;
  }
  close_entry(c, row, n, len, held);
}

// Blocks for each of n entries that share `pieces` pieces of work, `deep` of them a thread: eight
// blocks an SM in all (what is resident), no more than there is work for.
int spread(long long n, long long pieces, int deep, int sms) {
  const long long most = (pieces + kThreads * deep - 1) / (kThreads * deep);
  const long long want = (8LL * sms + n - 1) / n;
  const long long y = want < most ? want : most;
  return static_cast<int>(y < 1 ? 1 : y > 65535 ? 65535 : y);
}

}  // namespace

cudaError_t launch_cache_reset(const CacheView& c, int sms, cudaStream_t s) {
  reset_kernel<<<sms, kThreads, 0, s>>>(c);
  return cudaGetLastError();
}

cudaError_t launch_cache_free(const CacheView& c, int n, const int* seqs, cudaStream_t s) {
  free_kernel<<<n, kThreads, 0, s>>>(c, seqs);
  return cudaGetLastError();
}

cudaError_t launch_cache_reserve(const CacheView& c, int n, const int* seqs, const int* count, cudaStream_t s) {
  take_kernel<false><<<1, kTake, sizeof(int) * (n + 1), s>>>(c, n, seqs, count, nullptr, nullptr, nullptr);
  return cudaGetLastError();
}

cudaError_t launch_cache_fork(const CacheView& c, int n, const int* src, const int* dst, int* fresh, int* length,
                              int sms, cudaStream_t s) {
  take_kernel<true><<<1, kTake, sizeof(int) * (n + 1), s>>>(c, n, dst, nullptr, src, fresh, length);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const long long pieces = (2LL * c.layers * c.heads * c.row) << c.page_shift;
  return launch_chained(fork_kernel, dim3(n, spread(n, pieces / 2, kDeep, sms)), dim3(kThreads), 0, s, c, src, dst,
                        static_cast<const int*>(fresh), static_cast<const int*>(length));
}

cudaError_t launch_cache_append(const CacheView& c, const CacheAppend& a, int sms, cudaStream_t s) {
  const long long pieces = 2LL * a.layers * c.heads * c.row;
  append_kernel<<<dim3(static_cast<unsigned>(a.N), spread(a.N, pieces, 4, sms)), kThreads, 0, s>>>(c, a);
  return cudaGetLastError();
}

cudaError_t launch_cache_compact(const CacheView& c, int n, const int* seqs, const int* keep, const int* path,
                                 int path_ld, int sms, cudaStream_t s) {
  const long long pieces = 2LL * c.layers * c.heads * c.row;
  // Up to two pieces a thread one block moves as fast as two do, and needs no second kernel.
  if (path && pieces <= 2 * kThreads) {
    move_kernel<true><<<n, kThreads, 0, s>>>(c, seqs, keep, path, path_ld);
    return cudaGetLastError();
  }
  if (path) {
    move_kernel<false><<<dim3(n, spread(n, pieces, 1, sms)), kThreads, 0, s>>>(c, seqs, keep, path, path_ld);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_chained(close_kernel, dim3(n), dim3(kThreads), 0, s, c, seqs, keep, path, path_ld);
  }
  close_kernel<<<n, kThreads, 0, s>>>(c, seqs, keep, path, path_ld);
  return cudaGetLastError();
}

cudaError_t launch_cache_copy(const CacheView& from, const CacheView& to, int n, const int* src, const int* dst,
                              int sms, cudaStream_t s) {
  const long long pieces = (2LL * from.layers * from.heads * from.row) << from.page_shift;
  copy_kernel<<<dim3(n, spread(n, pieces, kDeep, sms)), kThreads, 0, s>>>(from, to, src, dst);
  return cudaGetLastError();
}

cudaError_t setup_cache_kernels() {
  const int bytes = sizeof(int) * (kCacheMaxEntries + 1);
  cudaError_t e = cudaFuncSetAttribute(take_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(take_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  return e;
}

}  // namespace mls
