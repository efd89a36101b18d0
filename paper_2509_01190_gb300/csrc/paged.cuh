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

struct PagedEntry {
  int keys, rows;  // keys of the entry, query rows per KV head
  int seq0;        // first sequence
};
__device__ __forceinline__ PagedEntry paged_entry(const PagedArgs& a, int e) {
  PagedEntry x;
  if (e < a.G) {
    x.seq0 = paged_group_at(a, e);
    x.rows = max(0, paged_group_at(a, e + 1) - x.seq0) * a.n_q * a.per;
    x.keys = min(max(a.plens[e], 0), a.pcols << a.page_shift);
  } else {
    x.seq0 = e - a.G;
    const bool live = a.G == 0 || (x.seq0 >= paged_group_at(a, 0) && x.seq0 < paged_group_at(a, a.G));
    x.rows = live ? a.n_q * a.per : 0;
    x.keys = max(0, min(a.lens[x.seq0], a.cols << a.page_shift) - (a.n_q - 1));
  }
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
// number t0.  CTA 0 also leaves what the joining kernel needs: the stretch length
// (0: nothing was done) and every entry's first block.  All NT threads; false: no work.
struct PagedSpan {
  int t, end, e, t0;
};
struct PagedPlanShared {
  long long warp[32];
  int e, t0;
};
template <int NT, int MT, int BN>
__device__ __forceinline__ bool paged_plan(const PagedArgs& a, const PagedWork& w, PagedPlanShared& sh, PagedSpan& s) {
  const int tid = threadIdx.x, lane = tid & 31;
  const int n = w.e1 - w.e0, q = (n + NT - 1) / NT;
  const int lo = min(n, tid * q), hi = min(n, lo + q);
  auto blocks = [&](int i) {
    const PagedEntry x = paged_entry(a, w.e0 + i);
    return static_cast<long long>(paged_blocks<BN>(x)) * paged_tiles<MT>(x) * a.Hkv;
  };
  long long sum = 0;
  for (int i = lo; i < hi; ++i) sum += blocks(i);
  long long upto = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) sh.warp[tid >> 5] = upto;
  __syncthreads();
  long long total = 0, before = 0;
#pragma unroll
  for (int k = 0; k < NT / 32; ++k) {
    if (k < (tid >> 5)) before += sh.warp[k];
    total += sh.warp[k];
  }
  // (group bounds that run backwards could pass any number of blocks)
  const bool sound = total <= 0x7fffffff - 0x100000;
  const long long per = max(static_cast<long long>(w.min_blocks), (total + gridDim.x - 1) / gridDim.x);
  const long long start = static_cast<long long>(blockIdx.x) * per;
  long long at = before + upto - sum;
  if (blockIdx.x == 0) {
    if (tid == 0) {
      w.head[0] = sound ? static_cast<int>(per) : 0;
      if (!sound) atomicOr(a.status, kStatusBadIndex);
    }
    long long f = at;
    for (int i = lo; i < hi; ++i) {
      w.head[1 + i] = static_cast<int>(f);
      f += blocks(i);
    }
  }
  if (!sound || start >= total) return false;
  if (start >= at && start < at + sum) {
    int i = lo;
    for (long long b = blocks(i); start >= at + b; b = blocks(i)) {
      at += b;
      ++i;
    }
    sh.e = w.e0 + i;
    sh.t0 = static_cast<int>(at);
  }
  __syncthreads();
  s.t = static_cast<int>(start);
  s.end = static_cast<int>(min(start + per, total));
  s.e = sh.e;
  s.t0 = sh.t0;
  return true;
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
    p.x = paged_entry(a, s.e);
    nb = paged_blocks<BN>(p.x);
    rt = paged_tiles<MT>(p.x);
    const int all = nb * rt * a.Hkv;
    if (s.t < s.t0 + all) break;
    s.t0 += all;
    ++s.e;
  }
  const int u = s.t - s.t0, item = u / nb;
  p.e = s.e;
  p.shared = s.e < a.G;
  p.h = item / rt;
  p.r = item % rt;
  p.b0 = u % nb;
  p.b1 = min(nb, p.b0 + s.end - s.t);
  p.slot = blockIdx.x + paged_first_item<MT>(a, w, p.x, s.e) + item;
  s.t += p.b1 - p.b0;
  return true;
}

// Page of entry i; a page number out of range is reported and page 0 read instead.
__device__ __forceinline__ int paged_page(const PagedArgs& a, const int32_t* row, int i) {
  int page = row[i >> a.page_shift];
  if (page < 0 || page >= a.n_pages) {
    atomicOr(a.status, kStatusBadIndex);
    page = 0;
  }
  return page;
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
