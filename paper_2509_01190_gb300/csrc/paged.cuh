// Work decomposition shared by the attention kernels over paged caches.
//
// The keys that every query of a call may see come in entries: the prefix of each
// group of sequences (its rows: the queries of all the group's sequences) and each
// sequence's own entries but for the last n_q - 1 (its rows: its own queries; the
// last n_q - 1 are hidden from some of them and belong to the joining kernel).  So
// no key of an entry is masked.  For each KV head the rows of an entry are cut into
// tiles of MT rows and its keys into blocks of BN; a tile's walk over its entry's
// blocks is an item.  All blocks of all items stand in one line, entry by entry, each
// item's behind `lead` units that stand for its start and end (which cost some blocks'
// time: without them the CTAs with the many short items would finish last by far),
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

// `given` entries of a table row with `cap` of them: a negative length counts as 0 (and nothing
// is taken off it that its type cannot hold)
__device__ __forceinline__ int paged_len(int given, int cap) { return min(max(given, 0), cap); }

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
  x.keys = max(0, paged_len(len, (shared ? a.pcols : a.cols) << a.page_shift) - (shared ? 0 : a.n_q - 1));
  return x;
}
// units of an entry for one tile of rows
template <int BN>
__device__ __forceinline__ int paged_units(const PagedWork& w, const PagedEntry& x) {
  return x.rows > 0 && x.keys > 0 ? (x.keys + BN - 1) / BN + w.lead : 0;
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

// This CTA's stretch [t, end) of the line; t lies in entry e, whose first unit is
// number t0.  The first warp works it out (its lanes over the entries; sums stop growing
// at kMostUnits, since group bounds that run backwards could pass any number) and tells
// the others; more warps would only queue for the same lines of L2.  CTA 0 also leaves
// what the joining kernel needs: the stretch length (0: nothing is done) and every entry's
// first unit.  All threads; false: no work.
struct PagedSpan {
  int t, end, e, t0;
  PagedLive live;
};
constexpr int kMostUnits = 0x3fffffff;
template <int MT, int BN>
__device__ __forceinline__ bool paged_plan(const PagedArgs& a, const PagedWork& w, PagedSpan& told, PagedSpan& s) {
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x, n = w.e1 - w.e0, q = (n + 31) / 32;
    const int lo = min(n, lane * q), hi = min(n, lo + q), grid = static_cast<int>(gridDim.x);
    const PagedLive live = paged_live(a);
    auto units = [&](int i) {
      const PagedEntry x = paged_entry(a, live, w.e0 + i);
      return paged_units<BN>(w, x) * paged_tiles<MT>(x) * a.Hkv;
    };
    int sum = 0;
#pragma unroll 2
    for (int i = lo; i < hi; ++i) sum = min(sum + units(i), kMostUnits);
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto = min(upto + v, kMostUnits);
    }
    const int total = __shfl_sync(0xffffffffu, upto, 31);
    const int per = max(w.min_units, static_cast<int>(static_cast<unsigned>(total + grid - 1) / static_cast<unsigned>(grid)));
    const int start = static_cast<int>(blockIdx.x) * per;
    const bool work = total < kMostUnits && start < total;
    int at = upto - sum;
    if (lane == 0) told.end = work ? min(start + per, total) : -1;
    if (work && start >= at && start < at + sum) {
      int i = lo;
      for (; i + 1 < hi; ++i) {
        const int n = units(i);
        if (start < at + n) break;
        at += n;
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
        at = min(at + units(i), kMostUnits);
      }
      if (lane == 0) {
        w.head[0] = total < kMostUnits ? per : 0;
        if (total >= kMostUnits) atomicOr(a.status, kStatusBadIndex);
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
  while (s.t < s.end) {
    p.x = paged_entry(a, s.live, s.e);
    const int nu = paged_units<BN>(w, p.x), rt = paged_tiles<MT>(p.x), all = nu * rt * a.Hkv;
    if (s.t >= s.t0 + all) {
      s.t0 += all;
      ++s.e;
      continue;
    }
    const unsigned u = static_cast<unsigned>(s.t - s.t0), item = u / static_cast<unsigned>(nu);
    const int u0 = static_cast<int>(u - item * static_cast<unsigned>(nu)), u1 = min(nu, u0 + s.end - s.t);
    s.t += u1 - u0;
    p.b0 = max(0, u0 - w.lead);
    p.b1 = u1 - w.lead;
    if (p.b0 >= p.b1) continue;  // no block of the item
    p.e = s.e;
    p.shared = s.e < a.G;
    p.h = rt == 1 ? item : item / static_cast<unsigned>(rt);
    p.r = static_cast<int>(item) - p.h * rt;
    p.slot = blockIdx.x + paged_first_item<MT>(a, w, p.x, s.e) + static_cast<int>(item);
    return true;
  }
  return false;
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
// The group of sequence s (the last one that starts at or before it): a lane per group, so
// one round trip for up to 32 groups; t0: first units of the entries, or null.  Whole warps.
struct PagedGroup {
  int g, seq0, end, keys, t0;  // g < 0: the sequence is padding
  bool beyond;                 // the prefix is longer than its table
};
__device__ __forceinline__ PagedGroup paged_group_of(const PagedArgs& a, int s, const int* t0) {
  const int lane = threadIdx.x & 31, end = paged_group_at(a, a.G), most = a.pcols << a.page_shift;
  PagedGroup r{-1, 0, 0, 0, 0, false};
  int len = 0;
  for (int i = 0; i < a.G; i += 32) {
    const int e = min(i + lane, a.G - 1);
    const int c0 = paged_group_at(a, e), c1 = paged_group_at(a, e + 1), pl = a.plens[e], pt = t0 != nullptr ? t0[e] : 0;
    const unsigned m = __ballot_sync(0xffffffffu, i + lane < a.G && c0 <= s);
    if (m == 0) break;
    const int src = 31 - __clz(m);
    r.g = i + src;
    r.seq0 = __shfl_sync(0xffffffffu, c0, src);
    r.end = __shfl_sync(0xffffffffu, c1, src);
    len = __shfl_sync(0xffffffffu, pl, src);
    r.t0 = __shfl_sync(0xffffffffu, pt, src);
  }
  if (s >= end) r.g = -1;
  r.keys = paged_len(len, most);
  r.beyond = len > most;
  return r;
}

// element offset, in q and out, of query row rr (of the entry's rows for head h)
template <int HD>
__device__ __forceinline__ size_t paged_q_at(const PagedArgs& a, const PagedPart& p, int rr) {
  const size_t tok = static_cast<size_t>(p.x.seq0) * a.n_q + rr / a.per;
  return (tok * (static_cast<size_t>(a.Hkv) * a.per) + static_cast<size_t>(p.h) * a.per + rr % a.per) * HD;
}

// N dims of a row in one load
template <typename T, int N>
__device__ __forceinline__ void paged_dims(const T* p, float (&x)[N]) {
  auto two = [&](int i, uint32_t y) {  // (bf16 is the upper half of a float)
    x[i] = __uint_as_float(y << 16);
    x[i + 1] = __uint_as_float(y & 0xffff0000u);
  };
  if constexpr (sizeof(T) == 4 && N == 4) {
    const float4 y = *reinterpret_cast<const float4*>(p);
    x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;
  } else if constexpr (sizeof(T) == 4 && N == 2) {
    const float2 y = *reinterpret_cast<const float2*>(p);
    x[0] = y.x, x[1] = y.y;
  } else if constexpr (sizeof(T) == 4) {
    x[0] = p[0];
  } else if constexpr (N == 4) {
    const uint2 y = *reinterpret_cast<const uint2*>(p);
    two(0, y.x);
    two(2, y.y);
  } else {
    two(0, *reinterpret_cast<const uint32_t*>(p));
  }
}

// The partial results of a query row from one launch: n of them, one slot after the other.
struct JoinParts {
  const float *o, *lse2;
  size_t step;  // rows from one slot to the next
  int n;
};
// rr: the row's number among its entry's rows for KV head g; per, t_entry: the stretch
// length and the entry's first unit
__device__ __forceinline__ JoinParts join_parts(const PagedArgs& a, const PagedWork& w, int e, const PagedEntry& x,
                                                int per, int t_entry, int g, int rr, int hd) {
  if (per == 0 || x.keys == 0) return JoinParts{nullptr, nullptr, 0, 0};
  const int ms = w.mt_shift, up = (1 << ms) - 1;
  const int nu = ((x.keys + (1 << w.bn_shift) - 1) >> w.bn_shift) + w.lead, rt = (x.rows + up) >> ms;
  const int item = g * rt + (rr >> ms), row = a.n_q * a.per;
  const unsigned t0 = static_cast<unsigned>(t_entry + item * nu);
  const int first = e < a.G ? (((x.seq0 * row) >> ms) + e) * a.Hkv
                            : (w.e0 < a.G ? (((a.S * row) >> ms) + a.G) * a.Hkv : 0) + x.seq0 * ((row + up) >> ms) * a.Hkv;
  const unsigned c0 = (t0 + w.lead) / static_cast<unsigned>(per), c1 = (t0 + nu - 1) / static_cast<unsigned>(per);  // (of its blocks)
  const size_t at = (static_cast<size_t>(static_cast<int>(c0) + first + item) << ms) + (rr & up);
  return JoinParts{w.o + at * hd, w.lse2 + at, static_cast<size_t>(1) << ms, static_cast<int>(c1 - c0) + 1};
}

// Those of row rr of sequence s, KV head g, from its group's prefix.
__device__ __forceinline__ JoinParts join_prefix(const PagedArgs& a, const PagedWork& w, const PagedGroup& x, int per, int s,
                                                 int g, int rr, int hd) {
  const PagedEntry e{x.keys, max(0, x.end - x.seq0) * a.n_q * a.per, x.seq0};
  rr += (s - x.seq0) * a.n_q * a.per;
  if ((threadIdx.x & 31) == 0 && (x.beyond || rr >= e.rows)) atomicOr(a.status, kStatusBadIndex);  // (bounds that run backwards)
  return rr < e.rows ? join_parts(a, w, x.g, e, per, x.t0, g, rr, hd) : JoinParts{nullptr, nullptr, 0, 0};
}

// Rows of one warp that belong to one sequence and KV head: maximum (log2), sum and result
// (not divided); a lane has DPL dims from DPL lane on.
template <int HD, int R>
struct PagedRows {
  int rr[R];  // row number among the sequence's n_q * per; below 0: none
  float m[R], l[R], acc[R][HD / 32];
};

// Adds each row's partial results of up to two launches, in the order of their keys: for 32
// of them the log2 sums, then the results, K of a row at a time.
template <typename T, int HD, int R, int K>
__device__ __forceinline__ void paged_add_parts(PagedRows<HD, R>& x, const JoinParts (&p)[R], const JoinParts (&p2)[R]) {
  constexpr int DPL = HD / 32;
  auto ex2 = [](float v) { return sizeof(T) == 4 ? exp2f(v) : ex2_fast(v); };
  const int lane = threadIdx.x & 31;
  int n = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) n = max(n, p[r].n + p2[r].n);
  for (int i0 = 0; i0 < n; i0 += 32) {
    float weight[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int i = i0 + lane, i2 = i - p[r].n;
      weight[r] = i2 < 0 ? p[r].lse2[i * p[r].step] : i2 < p2[r].n ? p2[r].lse2[i2 * p2[r].step] : -INFINITY;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float mn = fmaxf(x.m[r], warp_max(weight[r])), base = mn == -INFINITY ? 0.f : mn;
      const float f = ex2(x.m[r] - base);
      weight[r] = ex2(weight[r] - base);  // (0 past the last part; NaN stays NaN)
      x.m[r] = mn;
      x.l[r] = x.l[r] * f + warp_sum(weight[r]);
#pragma unroll
      for (int d = 0; d < DPL; ++d) x.acc[r][d] *= f;
    }
    const int most = min(32, n - i0);
    for (int k0 = 0; k0 < most; k0 += K) {
      float y[R][K][DPL];
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const int i = i0 + k0 + k, i2 = i - p[r].n;
#pragma unroll
          for (int d = 0; d < DPL; ++d) y[r][k][d] = 0.f;
          if (i2 < p2[r].n)
            paged_dims<float>((i2 < 0 ? p[r].o + i * p[r].step * HD : p2[r].o + i2 * p2[r].step * HD) + lane * DPL, y[r][k]);
        }
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const float e = __shfl_sync(0xffffffffu, weight[r], k0 + k);
#pragma unroll
          for (int d = 0; d < DPL; ++d) x.acc[r][d] = fmaf(e, y[r][k][d], x.acc[r][d]);
        }
    }
  }
}

// The end of rows of KV head g of sequence s, given what all of the sequence's queries see:
// adds the entries that a row's query sees and earlier ones do not, divides and writes.
template <typename T, int HD, int R>
__device__ __forceinline__ void paged_finish(const PagedArgs& a, int s, int g, PagedRows<HD, R>& x) {
  constexpr int DPL = HD / 32;
  auto ex2 = [](float v) { return sizeof(T) == 4 ? exp2f(v) : ex2_fast(v); };
  const int lane = threadIdx.x & 31, cap = a.cols << a.page_shift, given = a.lens[s], len = paged_len(given, cap);
  if (lane == 0 && given > cap) atomicOr(a.status, kStatusBadIndex);
  size_t row[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int rr = max(x.rr[r], 0), j = rr / a.per;
    row[r] = (static_cast<size_t>(s) * a.n_q + j) * (static_cast<size_t>(a.Hkv) * a.per) + g * a.per + rr - j * a.per;
  }
  if (a.n_q > 1) {
    const int first = max(0, len - a.n_q + 1);
    int n[R], most = 0;  // entries of a row, up to 16
    float q[R][DPL];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      n[r] = x.rr[r] < 0 ? 0 : len - a.n_q + x.rr[r] / a.per + 1 - first;
      most = max(most, n[r]);
      paged_dims<T>(static_cast<const T*>(a.q) + row[r] * HD + lane * DPL, q[r]);
    }
    const int pages = lane < most ? paged_page(a, a.table + static_cast<size_t>(s) * a.cols, first + lane) : 0;
    for (int i = 0; i < most; i += 4) {  // four entries a round trip
      float k4[4][DPL], v4[4][DPL];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int e = min(i + u, most - 1);
        const size_t at = paged_at<HD>(a, __shfl_sync(0xffffffffu, pages, e), g, first + e) + lane * DPL;
        paged_dims<T>(static_cast<const T*>(a.k) + at, k4[u]);
        paged_dims<T>(static_cast<const T*>(a.v) + at, v4[u]);
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (i >= n[r]) continue;
        float score[4], mn = x.m[r];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          score[u] = 0.f;
#pragma unroll
          for (int d = 0; d < DPL; ++d) score[u] = fmaf(q[r][d], k4[u][d], score[u]);
          score[u] = warp_sum(score[u]) * a.scale_log2;
          mn = i + u < n[r] ? fmaxf(mn, score[u]) : mn;
        }
        const float base = mn == -INFINITY ? 0.f : mn, f = ex2(x.m[r] - base);
        x.l[r] *= f;
#pragma unroll
        for (int d = 0; d < DPL; ++d) x.acc[r][d] *= f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (i + u < n[r]) {
            const float e = ex2(score[u] - base);
            x.l[r] += e;
#pragma unroll
            for (int d = 0; d < DPL; ++d) x.acc[r][d] = fmaf(e, v4[u][d], x.acc[r][d]);
          }
        x.m[r] = mn;
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (x.rr[r] < 0) continue;
    const float inv = x.l[r] > 0.f ? 1.f / x.l[r] : x.l[r];  // no key: zeros (NaN stays NaN)
    T* out = static_cast<T*>(a.out) + row[r] * HD + lane * DPL;
    const float(&o)[DPL] = x.acc[r];
    if constexpr (DPL == 4 && sizeof(T) == 2)
      *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
    else if constexpr (DPL == 2 && sizeof(T) == 2)
      *reinterpret_cast<uint32_t*>(out) = pack_bf16x2(o[0] * inv, o[1] * inv);
    else
#pragma unroll
      for (int d = 0; d < DPL; ++d) out[d] = from_f<T>(o[d] * inv);
    if (a.lse != nullptr && lane == 0) a.lse[row[r]] = x.m[r] + log2f(x.l[r]);
  }
}

}  // namespace zsaa
