// Work decomposition shared by the attention kernels over paged caches.
//
// The keys that every query of a call may see come in entries: the prefix of each
// group of sequences (its rows: the queries of all the group's sequences) and each
// sequence's own entries but for the last n_q - 1 (its rows: its own queries; the
// last n_q - 1 are hidden from some of them and belong to the joining kernel).  So
// no key of an entry is masked.  For each KV head the rows of an entry are cut into
// tiles of MT rows and its keys into blocks of BN; a tile's walk over its entry's
// blocks is an item.  All blocks of all items stand in one line, entry by entry,
// and every CTA takes an equal stretch of it, whatever the lengths are.  A stretch
// covers whole items or parts of them; for each it leaves one partial result
// (normalised rows and their log2 sums) in a slot, and the joining kernel adds a
// row's partials in the order of their keys, so results do not depend on timing.
//
// Slot: CTA number + item number.  Along the line either one or the other grows
// from a part to the next, so no two parts share a slot.  Item numbers need no
// scan: those of a group start at (rows of earlier groups / MT + group) * heads,
// which leaves room for each group's last, partly filled tile.
#pragma once

#include "common.cuh"
#include "paged.h"

namespace zsaa {

__device__ __forceinline__ float ex2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// first sequence of group g (numbers outside [0, S] are brought inside)
__device__ __forceinline__ int paged_group_at(const PagedArgs& a, int g) { return min(max(a.cu_seqs[g], 0), a.S); }

// the sequences that are not padding: [lo, hi)
struct PagedLive {
  int lo, hi;
};
__device__ __forceinline__ PagedLive paged_live(const PagedArgs& a) {
  if (a.G == 0) return PagedLive{0, a.S};
  return PagedLive{paged_group_at(a, 0), paged_group_at(a, a.G)};
}

struct PagedEntry {
  int keys, rows;  // keys of the entry, query rows per KV head
  int seq0;        // first sequence
};
// (loads first, and the same ones for either kind of entry: one round trip)
__device__ __forceinline__ PagedEntry paged_entry(const PagedArgs& a, const PagedLive& live, int e) {
  const bool shared = e < a.G;
  const int s = e - a.G;
  const int len = shared ? a.plens[e] : a.lens[s];
  int c0 = 0, c1 = 0;
  if (a.G > 0) {
    c0 = paged_group_at(a, min(e, a.G));
    c1 = paged_group_at(a, min(e + 1, a.G));
  }
  PagedEntry x;
  x.seq0 = shared ? c0 : s;
  x.rows = (shared ? max(0, c1 - c0) : s >= live.lo && s < live.hi ? 1 : 0) * a.n_q * a.per;
  x.keys = max(0, min(len, (shared ? a.pcols : a.cols) << a.page_shift) - (shared ? 0 : a.n_q - 1));
  return x;
}
// blocks of an entry for one tile of rows
template <int BN>
__device__ __forceinline__ int paged_blocks(const PagedEntry& x) {
  return x.rows > 0 ? (x.keys + BN - 1) / BN : 0;
}
template <int MT>
__device__ __forceinline__ int paged_tiles(const PagedEntry& x) { return (x.rows + MT - 1) / MT; }

// number of the entry's first item
template <int MT>
__device__ __forceinline__ int paged_first_item(const PagedArgs& a, const PagedWork& w, const PagedEntry& x, int e) {
  const int row = a.n_q * a.per;
  if (e < a.G) return (x.seq0 * row / MT + e) * a.Hkv;
  const int prefixes = w.e0 < a.G ? (a.S * row / MT + a.G) * a.Hkv : 0;
  return prefixes + x.seq0 * ((row + MT - 1) / MT) * a.Hkv;
}

// This CTA's stretch [t, end) of the line; t lies in entry e, whose first block is
// number t0.  The first warp works it out (its lanes over the entries; sums stop growing
// at kMostBlocks, since group bounds that run backwards could pass any number) and tells
// the others; more warps would only queue for the same lines of L2.  CTA 0 also leaves
// what the joining kernel needs: the stretch length (0: nothing is done) and every entry's
// first block.  All threads; false: no work.
struct PagedSpan {
  int t, end, e, t0;
  PagedLive live;
};
constexpr int kMostBlocks = 0x3fffffff;
template <int MT, int BN>
__device__ __forceinline__ bool paged_plan(const PagedArgs& a, const PagedWork& w, PagedSpan& told, PagedSpan& s) {
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x, n = w.e1 - w.e0, q = (n + 31) / 32;
    const int lo = min(n, lane * q), hi = min(n, lo + q), grid = static_cast<int>(gridDim.x);
    const PagedLive live = paged_live(a);
    auto blocks = [&](int i) {
      const PagedEntry x = paged_entry(a, live, w.e0 + i);
      return paged_blocks<BN>(x) * paged_tiles<MT>(x) * a.Hkv;
    };
    int sum = 0;
#pragma unroll 2
    for (int i = lo; i < hi; ++i) sum = min(sum + blocks(i), kMostBlocks);
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto = min(upto + v, kMostBlocks);
    }
    const int total = __shfl_sync(0xffffffffu, upto, 31);
    const int per = max(w.min_blocks, static_cast<int>(static_cast<unsigned>(total + grid - 1) / static_cast<unsigned>(grid)));
    const int start = static_cast<int>(blockIdx.x) * per;
    const bool work = total < kMostBlocks && start < total;
    int at = upto - sum;
    if (lane == 0) told.end = work ? min(start + per, total) : -1;
    if (work && start >= at && start < at + sum) {
      int i = lo;
      for (; i + 1 < hi; ++i) {
        const int b = blocks(i);
        if (start < at + b) break;
        at += b;
      }
      told.t = start;
      told.e = w.e0 + i;
      told.t0 = at;
      told.live = live;
    }
    if (blockIdx.x == 0) {
      at = upto - sum;
      for (int i = lo; i < hi; ++i) {
        w.head[1 + i] = at;
        at = min(at + blocks(i), kMostBlocks);
      }
      if (lane == 0) {
        w.head[0] = total < kMostBlocks ? per : 0;
        if (total >= kMostBlocks) atomicOr(a.status, kStatusBadIndex);
      }
    }
  }
  __syncthreads();
  s = told;
  return s.end >= 0;
}

// The next part of the stretch: one tile of rows of one head over blocks [b0, b1).
struct PagedPart {
  PagedEntry x;
  int e, h, r, b0, b1;
  int slot;
  bool shared;  // a prefix
};
template <int MT, int BN>
__device__ __forceinline__ bool paged_next(const PagedArgs& a, const PagedWork& w, PagedSpan& s, PagedPart& p) {
  if (s.t >= s.end) return false;
  int nb, rt;
  while (true) {
    p.x = paged_entry(a, s.live, s.e);
    nb = paged_blocks<BN>(p.x);
    rt = paged_tiles<MT>(p.x);
    const int all = nb * rt * a.Hkv;
    if (s.t < s.t0 + all) break;
    s.t0 += all;
    ++s.e;
  }
  const unsigned u = static_cast<unsigned>(s.t - s.t0), item = u / static_cast<unsigned>(nb);
  p.e = s.e;
  p.shared = s.e < a.G;
  p.h = rt == 1 ? item : item / static_cast<unsigned>(rt);
  p.r = static_cast<int>(item) - p.h * rt;
  p.b0 = static_cast<int>(u - item * static_cast<unsigned>(nb));
  p.b1 = min(nb, p.b0 + s.end - s.t);
  p.slot = blockIdx.x + paged_first_item<MT>(a, w, p.x, s.e) + static_cast<int>(item);
  s.t += p.b1 - p.b0;
  return true;
}

// A page number out of range is reported, and page 0 read instead.
__device__ __forceinline__ int paged_sound(const PagedArgs& a, int page) {
  if (page < 0 || page >= a.n_pages) {
    atomicOr(a.status, kStatusBadIndex);
    page = 0;
  }
  return page;
}
// Page of entry i
__device__ __forceinline__ int paged_page(const PagedArgs& a, const int32_t* row, int i) {
  return paged_sound(a, row[i >> a.page_shift]);
}
__device__ __forceinline__ const int32_t* paged_row(const PagedArgs& a, const PagedPart& p) {
  return p.shared ? a.ptable + static_cast<size_t>(p.e) * a.pcols : a.table + static_cast<size_t>(p.x.seq0) * a.cols;
}
// element offset of entry i of KV head h
template <int HD>
__device__ __forceinline__ size_t paged_at(const PagedArgs& a, int page, int h, int i) {
  return (((static_cast<size_t>(page) * a.Hkv + h) << a.page_shift) + (i & ((1 << a.page_shift) - 1))) * HD;
}
// element offset, in q and out, of query row rr (of the entry's rows for head h)
template <int HD>
__device__ __forceinline__ size_t paged_q_at(const PagedArgs& a, const PagedPart& p, int rr) {
  const size_t tok = static_cast<size_t>(p.x.seq0) * a.n_q + rr / a.per;
  return (tok * (static_cast<size_t>(a.Hkv) * a.per) + static_cast<size_t>(p.h) * a.per + rr % a.per) * HD;
}

}  // namespace zsaa
