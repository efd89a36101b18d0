// Pages counted by reference: tables that grow and shrink (resize), sequences that continue
// others (fork), and entries moved together (compact).
//
// refs[page] counts the table entries that name a page; a page with none is free, and there is
// no other list of free pages.  A call that needs pages takes those of the lowest numbers, in
// the order of its rows and columns: what it takes follows from the counts alone, not from
// timing, although the counts themselves change by atomics (whose order does not matter).
#include <algorithm>

#include "common.cuh"
#include "paged.h"

namespace zsaa {
namespace {

// As launch_kernel, in clusters of `ctas` along x.
template <typename... KArgs, typename... Args>
cudaError_t launch_cluster(void (*kernel)(KArgs...), dim3 grid, dim3 block, int ctas, size_t smem, cudaStream_t s, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ctas > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

// ---------------------------------------------------------------- taking and giving up pages

// One cluster does a call: its CTAs change the counts, meet, count the free pages of their
// parts of the pool, exchange the counts, and hand out the pages.
constexpr int kTakeThreads = 1024, kTakeWarps = kTakeThreads / 32, kTakeCtas = 8;
constexpr int kTakeBlock = 128;  // columns of a table row that a warp looks at together
constexpr int kTakeMasks = 64;   // words of free pages that a warp keeps

// pages of a warp's part of the pool
__host__ __device__ inline int pages_part(int n_pages, int warps) { return ((n_pages + warps - 1) / warps + 31) & ~31; }

// What a call does with one row of its table.
struct TakeRow {
  int touch0, touch1;  // columns given up (resize) or shared (fork)
  int first, need;     // columns that get a new page: [first, first + need)
  int goal, least;     // the length with all of its new pages, and with none of them
  int src;             // fork: the parent's row, or -1
  bool bad;
};

__device__ __forceinline__ int pages_of(int n, int shift) {
  return static_cast<int>((static_cast<unsigned>(n) + ((1u << shift) - 1)) >> shift);
}

template <bool FORK>
__device__ __forceinline__ TakeRow take_row(const PagesArgs& a, int i) {
  TakeRow r{};
  const int cap = a.cols << a.page_shift;
  if constexpr (FORK) {
    const int p = a.parent[i];
    r.src = p >= 0 && p < a.parents ? p : -1;
    r.bad = p < -1 || p >= a.parents;
    const int given = r.src >= 0 ? a.lens[r.src] : 0;
    r.bad |= given > cap;
    int len = min(max(given, 0), cap);
    if (a.at != nullptr && r.src >= 0) len = min(len, max(a.at[i], 0));
    const int whole = len >> a.page_shift;
    r.touch1 = r.first = whole;
    r.need = (len & ((1 << a.page_shift) - 1)) != 0;
    r.goal = len;
    r.least = whole << a.page_shift;
  } else {
    const int had = a.lens[i], wants = a.want[i];
    r.bad = had > cap || wants > cap;
    const int len = min(max(had, 0), cap), goal = min(max(wants, 0), cap);
    const int held = pages_of(len, a.page_shift), to = pages_of(goal, a.page_shift);
    r.touch0 = min(to, held);
    r.touch1 = held;
    r.first = held;
    r.need = max(to - held, 0);
    r.goal = goal;
    r.least = r.need > 0 ? held << a.page_shift : goal;
  }
  return r;
}

__device__ __forceinline__ void st_cluster_u32(uint32_t saddr, uint32_t rank, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_rank(saddr, rank)), "r"(v) : "memory");
}

template <bool FORK>
__global__ void __launch_bounds__(kTakeThreads, 1) pages_take_kernel(const __grid_constant__ PagesArgs given) {
  extern __shared__ int dynamic[];
  __shared__ int warp_sum[kTakeWarps], warp_free[kTakeWarps], cta_free[kTakeCtas];
  pdl_trigger();
  PagesArgs a = given;
  int* base = dynamic;             // [rows + 1]: pages that earlier rows need
  int* touch = base + a.rows + 1;  // [rows]: first column given up or shared
  int* end = touch + a.rows;       // [rows]: the column behind the last; the first that gets a page
  unsigned* masks = reinterpret_cast<unsigned*>(end + a.rows);  // free pages of a warp's part, 32 to a word
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = static_cast<int>(cluster_rank()), ctas = static_cast<int>(cluster_size());
  const int gw = rank * kTakeWarps + warp, warps = ctas * kTakeWarps;
  pdl_wait();
  a.refs = after_wait(a.refs), a.table = after_wait(a.table), a.lens = after_wait(a.lens);
  if (FORK) a.parent = after_wait(a.parent), a.at = after_wait(a.at);
  else a.want = after_wait(a.want);

  // the rows, every CTA for itself: what each gives up or shares, and the pages needed before it
  const int own = rank * kTakeThreads + tid;  // the row whose length this thread writes (the first one)
  TakeRow own_row{};
  const int per = (a.rows + kTakeThreads - 1) / kTakeThreads, i0 = min(tid * per, a.rows), i1 = min(i0 + per, a.rows);
  int mine = 0;
  for (int i = i0; i < i1; ++i) {
    const TakeRow r = take_row<FORK>(a, i);
    mine += r.need;
    touch[i] = r.touch0;
    end[i] = r.first;
    base[i] = r.need;
    if (r.bad && rank == 0) atomicOr(a.status, kStatusBadIndex);
  }
  if (own < a.rows) own_row = take_row<FORK>(a, own);
  int run = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += x;
  }
  if (lane == 31) warp_sum[warp] = run;
  __syncthreads();
  int before = run - mine, total_need = 0;
#pragma unroll
  for (int w = 0; w < kTakeWarps; ++w) {
    before += w < warp ? warp_sum[w] : 0;
    total_need += warp_sum[w];
  }
  for (int i = i0; i < i1; ++i) {
    const int need = base[i];
    base[i] = before;
    before += need;
  }
  if (tid == 0) base[a.rows] = total_need;

  // pages given up or shared.  (A count that falls below 0 is found with the free pages.)
  const int blocks = (a.cols + kTakeBlock - 1) / kTakeBlock;
  const long long units = static_cast<long long>(a.rows) * blocks;
#pragma unroll 2
  for (long long u = gw; u < units; u += warps) {
    const int i = static_cast<int>(u / blocks), c0 = static_cast<int>(u - static_cast<long long>(i) * blocks) * kTakeBlock;
    const int t0 = touch[i], t1 = end[i];
    if (t0 >= c0 + kTakeBlock || t1 <= c0) continue;
    const int32_t* row = a.table + static_cast<size_t>(FORK ? a.parent[i] : i) * a.cols;
    int page[kTakeBlock / 32];
#pragma unroll
    for (int k = 0; k < kTakeBlock / 32; ++k) {
      const int c = c0 + 32 * k + lane;
      page[k] = c >= t0 && c < t1 ? row[c] : -1;
    }
#pragma unroll
    for (int k = 0; k < kTakeBlock / 32; ++k) {
      const int c = c0 + 32 * k + lane;
      if (c < t0 || c >= t1) continue;
      if (FORK) a.table_out[static_cast<size_t>(i) * a.cols + c] = page[k];
      if (page[k] < 0 || page[k] >= a.n_pages) atomicOr(a.status, kStatusBadIndex);
      else atomicAdd(a.refs + page[k], FORK ? 1 : -1);
    }
  }
  __threadfence();
  cluster_sync_all();

  // the free pages of this warp's part of the pool
  const int part = pages_part(a.n_pages, warps), words = part / 32;
  const bool kept = words <= kTakeMasks;
  const long long p0 = static_cast<long long>(gw) * part;
  const int q0 = static_cast<int>(min(p0, static_cast<long long>(a.n_pages)));
  const int q1 = static_cast<int>(min(p0 + part, static_cast<long long>(a.n_pages)));
  auto free_of = [&](int q) {
    const int c = q + lane < q1 ? __ldcg(a.refs + q + lane) : 1;
    if (c < 0) {  // more given up than there were
      a.refs[q + lane] = 0;
      atomicOr(a.status, kStatusBadIndex);
    }
    return __ballot_sync(0xffffffffu, c <= 0);
  };
  int n_free = 0;
#pragma unroll 8
  for (int w = 0; w < words; ++w) {
    const int q = q0 + 32 * w;
    if (q >= q1) break;
    const unsigned m = free_of(q);
    if (kept && lane == 0) masks[warp * words + w] = m;
    n_free += __popc(m);
  }
  if (lane == 0) warp_free[warp] = n_free;
  __syncthreads();
  int free_before = 0, cta_total = 0;
#pragma unroll
  for (int w = 0; w < kTakeWarps; ++w) {
    free_before += w < warp ? warp_free[w] : 0;
    cta_total += warp_free[w];
  }
  if (tid < ctas) st_cluster_u32(smem_u32(&cta_free[rank]), tid, cta_total);
  cluster_sync_all();
  int free_total = 0;
  for (int r = 0; r < ctas; ++r) {
    free_before += r < rank ? cta_free[r] : 0;
    free_total += cta_free[r];
  }

  // the free page of rank k goes to the k-th place that needs one
#pragma unroll 2
  for (int w = 0; w < words; ++w) {
    const int q = q0 + 32 * w;
    if (q >= q1 || free_before >= total_need) break;
    const unsigned mask = kept ? masks[warp * words + w] : free_of(q);
    const int k = free_before + __popc(mask & ((1u << lane) - 1));
    free_before += __popc(mask);
    if ((mask >> lane & 1) == 0 || k >= total_need) continue;
    int lo = 0, hi = a.rows;  // base[lo] <= k < base[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (base[mid] <= k) lo = mid; else hi = mid;
    }
    a.table_out[static_cast<size_t>(lo) * a.cols + end[lo] + (k - base[lo])] = q + lane;
    a.refs[q + lane] = 1;
  }
  for (int i = own; i < a.rows; i += ctas * kTakeThreads) {
    const TakeRow r = i == own ? own_row : take_row<FORK>(a, i);
    const int got = min(max(free_total - base[i], 0), r.need);
    // (the last page may be needed in part)
    a.lens_out[i] = got == r.need ? r.goal : r.least + (got << a.page_shift);
  }
  if (given.n_free != nullptr && rank == 0 && tid == 0) *given.n_free = free_total - min(free_total, total_need);
}

template <bool FORK>
cudaError_t run_take(const PagesArgs& a, cudaStream_t s) {
  const int words = pages_part(a.n_pages, kTakeCtas * kTakeWarps) / 32;
  const size_t smem = sizeof(int) * (3 * static_cast<size_t>(a.rows) + 1 + (words <= kTakeMasks ? words * kTakeWarps : 0));
  static OncePerDevice once;
  const cudaError_t e = set_smem_limit_once(once, pages_take_kernel<FORK>,
                                            static_cast<int>(sizeof(int)) * (3 * kPagesMaxRows + 1 + kTakeMasks * kTakeWarps));
  if (e != cudaSuccess) return e;
  return launch_cluster(pages_take_kernel<FORK>, dim3(kTakeCtas), dim3(kTakeThreads), kTakeCtas, smem, s, a);
}

// ---------------------------------------------------------------- fork: the partly filled pages

struct ForkCopyArgs {
  PoolList pools;
  const int32_t *table, *table_out, *parent, *lens_out;
  int cols, n_pages, page_shift, Hkv, row_vecs;
  int* status;
};

__global__ void __launch_bounds__(256) fork_copy_kernel(const __grid_constant__ ForkCopyArgs a) {
  pdl_trigger();
  pdl_wait();
  const int i = blockIdx.x, tid = threadIdx.x;
  const int len = after_wait(a.lens_out)[i];
  const int whole = len >> a.page_shift, part = len & ((1 << a.page_shift) - 1);
  if (part == 0) return;
  const int from = after_wait(a.table)[static_cast<size_t>(after_wait(a.parent)[i]) * a.cols + whole];
  const int to = after_wait(a.table_out)[static_cast<size_t>(i) * a.cols + whole];
  if (from < 0 || from >= a.n_pages) {
    if (tid == 0) atomicOr(a.status, kStatusBadIndex);
    return;
  }
  const int n = part * a.row_vecs, stride = a.row_vecs << a.page_shift;  // vectors to copy, and of a page, per head
  uint4* pool = static_cast<uint4*>(a.pools.p[blockIdx.y]);
  const uint4* s = pool + static_cast<size_t>(from) * a.Hkv * stride;
  uint4* d = pool + static_cast<size_t>(to) * a.Hkv * stride;
  for (int h = 0; h < a.Hkv; ++h)
    for (int v = tid; v < n; v += blockDim.x) d[static_cast<size_t>(h) * stride + v] = s[static_cast<size_t>(h) * stride + v];
}

// ---------------------------------------------------------------- compact

// A cluster of CTAs (often one) moves some heads' entries of one sequence in one pool, a tile of
// entries after the other: the tile's loads, a barrier of the cluster, its stores.  Entry start + j
// comes from keep[j] >= start + j, so what a tile writes is never read by a later one, and in
// place is as right as into other pages.  While a tile's values are on their way the next tile's
// places are looked up (keep -> table -> page, three round trips), so a tile costs about one
// round trip.
constexpr int kCompactThreads = 256, kCompactUnroll = 8, kCompactVecs = kCompactThreads * kCompactUnroll;

struct CompactPlan {
  int heads;  // of a CTA
  int tile;   // entries of a CTA's share of a tile: heads * tile * row_vecs <= kCompactVecs
  int ctas;   // of a cluster
};

__global__ void __launch_bounds__(kCompactThreads, 3)
    compact_kernel(const __grid_constant__ CompactArgs a, const __grid_constant__ PoolList pools, const __grid_constant__ CompactPlan plan) {
  __shared__ int s_from[2][kCompactVecs / 8], s_to[2][kCompactVecs / 8];  // entries in the pool (of head 0), or -1
  pdl_trigger();
  pdl_wait();
  const int rank = static_cast<int>(blockIdx.x) % plan.ctas, s = static_cast<int>(blockIdx.x) / plan.ctas, tid = threadIdx.x;
  const int h0 = blockIdx.z * plan.heads, heads = min(plan.heads, a.Hkv - h0);
  const bool first_cta = blockIdx.y == 0 && h0 == 0;
  const int given = after_wait(a.lens)[s], cap = a.cols << a.page_shift, out_cap = a.out_cols << a.page_shift;
  const int len = min(max(given, 0), cap);
  const int begin = a.start != nullptr ? after_wait(a.start)[s] : 0, start = min(max(begin, 0), len);
  const int listed = after_wait(a.n_keep)[s];
  const int n = min(min(max(listed, 0), a.keep_cols), min(len, out_cap) - min(start, out_cap));
  if (first_cta && rank == 0 && tid == 0) {
    a.lens_out[s] = start + n;
    if (given > cap || begin > len || listed > n) atomicOr(a.status, kStatusBadIndex);
  }
  const int32_t* keep = after_wait(a.keep) + static_cast<size_t>(s) * a.keep_cols;
  const int32_t* from_row = after_wait(a.table) + static_cast<size_t>(s) * a.cols;
  const int32_t* to_row = after_wait(a.table_out) + static_cast<size_t>(s) * a.out_cols;
  const int mask = (1 << a.page_shift) - 1, step = plan.tile * plan.ctas;
  // this CTA's entries of the tile from j0 on
  auto look_up = [&](unsigned j0, int slot) {  // (j0 may pass 2^31)
    for (int i = tid; i < plan.tile; i += kCompactThreads) {
      const unsigned j = j0 + rank * plan.tile + i;
      int from = -1, to = -1;
      if (j < static_cast<unsigned>(n)) {
        const int e = keep[j], d = start + static_cast<int>(j);
        const int before = j > 0 ? keep[j - 1] : -1, q = to_row[d >> a.page_shift];
        bool ok = e >= d && e < len && before < e;
        const int p = ok ? from_row[e >> a.page_shift] : -1;
        ok = p >= 0 && p < a.n_pages && q >= 0 && q < a.n_pages;
        const bool stays = p == q && e == d;
        if (ok && !stays && a.refs != nullptr) ok = after_wait(a.refs)[q] == 1;  // no other sequence's page
        if (!ok && first_cta) atomicOr(a.status, kStatusBadIndex);
        if (ok && !stays) {
          from = ((p * a.Hkv) << a.page_shift) + (e & mask);
          to = ((q * a.Hkv) << a.page_shift) + (d & mask);
        }
      }
      s_from[slot][i] = from;
      s_to[slot][i] = to;
    }
  };
  uint4* pool = static_cast<uint4*>(pools.p[blockIdx.y]);
  const int row_shift = 31 - __clz(a.row_vecs), vec = tid & (a.row_vecs - 1);
  const int at = tid >> row_shift, rows = kCompactThreads >> row_shift;  // (head, entry) pairs of a round
  look_up(0, 0);
  __syncthreads();
  int slot = 0;
  for (unsigned j0 = 0; j0 < static_cast<unsigned>(n); j0 += step, slot ^= 1) {
    uint4 x[kCompactUnroll];
    int to[kCompactUnroll];
#pragma unroll
    for (int k = 0; k < kCompactUnroll; ++k) {
      const int i = k * rows + at, h = i / plan.tile, e = i - h * plan.tile;
      to[k] = -1;
      if (h >= heads) continue;
      const int from = s_from[slot][e], head = (h0 + h) << a.page_shift;
      if (from < 0) continue;
      x[k] = pool[(static_cast<size_t>(from + head) << row_shift) + vec];
      to[k] = s_to[slot][e] + head;
    }
    if (j0 + step < static_cast<unsigned>(n)) look_up(j0 + step, slot ^ 1);
    if (plan.ctas > 1) cluster_sync_all(); else __syncthreads();
#pragma unroll
    for (int k = 0; k < kCompactUnroll; ++k)
      if (to[k] >= 0) pool[(static_cast<size_t>(to[k]) << row_shift) + vec] = x[k];
  }
}

// A CTA takes as many heads as its registers hold of the longest list, and clusters split a list
// where its CTAs would not fill the SMs.
CompactPlan compact_plan(const CompactArgs& a, int pools, int sms) {
  CompactPlan p{1, kCompactVecs / a.row_vecs, 1};
  p.tile = std::min(p.tile, a.keep_cols);
  p.heads = std::max(1, std::min(a.Hkv, kCompactVecs / (a.row_vecs * p.tile)));
  const long long ctas = static_cast<long long>(a.S) * pools * ((a.Hkv + p.heads - 1) / p.heads);
  while (p.ctas < 8 && ctas * p.ctas < 2 * sms && p.tile * p.ctas < a.keep_cols) p.ctas *= 2;
  return p;
}

}  // namespace

cudaError_t launch_paged_resize(const PagesArgs& a, cudaStream_t s) { return run_take<false>(a, s); }

cudaError_t launch_paged_fork(const PagesArgs& a, const PoolList& pools, int Hkv, int row_vecs, cudaStream_t s) {
  const cudaError_t e = run_take<true>(a, s);
  if (e != cudaSuccess) return e;
  ForkCopyArgs c{};
  c.pools = pools;
  c.table = a.table, c.table_out = a.table_out, c.parent = a.parent, c.lens_out = a.lens_out;
  c.cols = a.cols, c.n_pages = a.n_pages, c.page_shift = a.page_shift, c.Hkv = Hkv, c.row_vecs = row_vecs;
  c.status = a.status;
  ZSAA_LAUNCH(fork_copy_kernel, dim3(a.rows, pools.n), dim3(256), 0, s, c);
  return cudaSuccess;
}

cudaError_t launch_paged_compact(const CompactArgs& a, const PoolList& pools, int sms, cudaStream_t s) {
  const CompactPlan p = compact_plan(a, pools.n, sms);
  return launch_cluster(compact_kernel, dim3(a.S * p.ctas, pools.n, (a.Hkv + p.heads - 1) / p.heads), dim3(kCompactThreads),
                        p.ctas, 0, s, a, pools, p);
}

}  // namespace zsaa
