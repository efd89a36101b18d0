// Pages counted by reference: tables that grow and shrink (resize), sequences that continue
// others (fork), and entries moved together (compact).
//
// refs[page] counts the table entries that name a page; a page with none is free, and there is
// no other list of free pages.  A call that needs pages takes those of the lowest numbers, in
// the order of its rows and columns: what it takes follows from the counts alone, not from
// timing, although the counts themselves change by atomics (whose order does not matter).
#include "common.cuh"
#include "paged.h"

namespace zsaa {
namespace {

// ---------------------------------------------------------------- taking and giving up pages

// One cluster does a call: its CTAs change the counts, meet, count the free pages of their
// parts of the pool, exchange the counts, and hand out the pages.
constexpr int kTakeThreads = 1024, kTakeWarps = kTakeThreads / 32, kTakeCtas = 8;
constexpr int kTakeBlock = 128;  // columns of a table row that a warp looks at together

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
  extern __shared__ int base[];  // [rows + 1]: pages that earlier rows need
  __shared__ int warp_sum[kTakeWarps], warp_free[kTakeWarps], cta_free[kTakeCtas];
  pdl_trigger();
  pdl_wait();
  PagesArgs a = given;
  a.refs = after_wait(a.refs), a.table = after_wait(a.table), a.lens = after_wait(a.lens);
  if (FORK) a.parent = after_wait(a.parent), a.at = after_wait(a.at);
  else a.want = after_wait(a.want);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = static_cast<int>(cluster_rank()), ctas = static_cast<int>(cluster_size());
  const int gw = rank * kTakeWarps + warp, warps = ctas * kTakeWarps;

  // pages given up or shared
  const int blocks = (a.cols + kTakeBlock - 1) / kTakeBlock;
  const long long units = static_cast<long long>(a.rows) * blocks;
  for (long long u = gw; u < units; u += warps) {
    const int i = static_cast<int>(u / blocks), c0 = static_cast<int>(u % blocks) * kTakeBlock;
    const TakeRow r = take_row<FORK>(a, i);
    if (r.bad && c0 == 0 && lane == 0) atomicOr(a.status, kStatusBadIndex);
    if (r.touch0 >= c0 + kTakeBlock || r.touch1 <= c0) continue;
    const int32_t* row = a.table + static_cast<size_t>(FORK ? r.src : i) * a.cols;
    int page[kTakeBlock / 32];
#pragma unroll
    for (int k = 0; k < kTakeBlock / 32; ++k) {
      const int c = c0 + 32 * k + lane;
      page[k] = c >= r.touch0 && c < r.touch1 ? row[c] : -1;
    }
#pragma unroll
    for (int k = 0; k < kTakeBlock / 32; ++k) {
      const int c = c0 + 32 * k + lane;
      if (c < r.touch0 || c >= r.touch1) continue;
      if (FORK) a.table_out[static_cast<size_t>(i) * a.cols + c] = page[k];
      if (page[k] < 0 || page[k] >= a.n_pages) {
        atomicOr(a.status, kStatusBadIndex);
      } else if (FORK) {
        atomicAdd(a.refs + page[k], 1);
      } else if (atomicSub(a.refs + page[k], 1) <= 0) {  // a page that nothing refers to
        atomicAdd(a.refs + page[k], 1);
        atomicOr(a.status, kStatusBadIndex);
      }
    }
  }
  __threadfence();
  cluster_sync_all();

  // pages needed before each row (every CTA for itself)
  const int per = (a.rows + kTakeThreads - 1) / kTakeThreads, i0 = min(tid * per, a.rows), i1 = min(i0 + per, a.rows);
  int mine = 0;
  for (int i = i0; i < i1; ++i) mine += take_row<FORK>(a, i).need;
  int run = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += x;
  }
  if (lane == 31) warp_sum[warp] = run;
  // free pages of this warp's part of the pool
  const int part = ((a.n_pages + warps - 1) / warps + 31) & ~31;
  const long long p0 = static_cast<long long>(gw) * part;
  const int q0 = static_cast<int>(min(p0, static_cast<long long>(a.n_pages)));
  const int q1 = static_cast<int>(min(p0 + part, static_cast<long long>(a.n_pages)));
  int n_free = 0;
#pragma unroll 4
  for (int q = q0; q < q1; q += 32) n_free += q + lane < q1 && __ldcg(a.refs + q + lane) == 0;
  n_free = __reduce_add_sync(0xffffffffu, n_free);
  if (lane == 0) warp_free[warp] = n_free;
  __syncthreads();
  int before = 0, total_need = 0, free_before = 0, cta_total = 0;
#pragma unroll
  for (int w = 0; w < kTakeWarps; ++w) {
    before += w < warp ? warp_sum[w] : 0;
    total_need += warp_sum[w];
    free_before += w < warp ? warp_free[w] : 0;
    cta_total += warp_free[w];
  }
  before += run - mine;
  for (int i = i0; i < i1; ++i) {
    base[i] = before;
    before += take_row<FORK>(a, i).need;
  }
  if (tid == 0) base[a.rows] = total_need;
  if (tid < ctas) st_cluster_u32(smem_u32(&cta_free[rank]), tid, cta_total);
  cluster_sync_all();
  int free_total = 0;
  for (int r = 0; r < ctas; ++r) {
    free_before += r < rank ? cta_free[r] : 0;
    free_total += cta_free[r];
  }

  // the free page of rank k goes to the k-th place that needs one
  for (int q = q0; q < q1 && free_before < total_need; q += 32) {
    const bool is_free = q + lane < q1 && __ldcg(a.refs + q + lane) == 0;
    const unsigned mask = __ballot_sync(0xffffffffu, is_free);
    const int k = free_before + __popc(mask & ((1u << lane) - 1));
    free_before += __popc(mask);
    if (!is_free || k >= total_need) continue;
    int lo = 0, hi = a.rows;  // base[lo] <= k < base[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (base[mid] <= k) lo = mid; else hi = mid;
    }
    const int c = take_row<FORK>(a, lo).first + (k - base[lo]);
    a.table_out[static_cast<size_t>(lo) * a.cols + c] = q + lane;
    a.refs[q + lane] = 1;
  }
  for (int i = rank * kTakeThreads + tid; i < a.rows; i += ctas * kTakeThreads) {
    const TakeRow r = take_row<FORK>(a, i);
    const int got = min(max(free_total - base[i], 0), r.need);
    // (the last page may be needed in part)
    a.lens_out[i] = got == r.need ? r.goal : r.least + (got << a.page_shift);
  }
  if (given.n_free != nullptr && rank == 0 && tid == 0) *given.n_free = free_total - min(free_total, total_need);
}

template <bool FORK>
cudaError_t run_take(const PagesArgs& a, cudaStream_t s) {
  const size_t smem = sizeof(int) * (static_cast<size_t>(a.rows) + 1);
  static OncePerDevice once;
  const cudaError_t e = set_smem_limit_once(once, pages_take_kernel<FORK>, sizeof(int) * (kPagesMaxRows + 1));
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kTakeCtas);
  cfg.blockDim = dim3(kTakeThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kTakeCtas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, pages_take_kernel<FORK>, a);
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

// One CTA moves one head's entries of one sequence in one pool, a tile of entries after the
// other: the loads of a tile, a barrier, its stores.  Entry start + j comes from keep[j] >=
// start + j, so a tile's places are never read by a later tile, and in place is as right as
// into other pages.
constexpr int kCompactThreads = 256, kCompactUnroll = 8;

__global__ void __launch_bounds__(kCompactThreads) compact_kernel(const __grid_constant__ CompactArgs a,
                                                                  const __grid_constant__ PoolList pools) {
  pdl_trigger();
  pdl_wait();
  const int s = blockIdx.x, h = blockIdx.z, tid = threadIdx.x;
  const bool head = blockIdx.y == 0 && h == 0;
  const int given = after_wait(a.lens)[s], cap = a.cols << a.page_shift, out_cap = a.out_cols << a.page_shift;
  const int len = min(max(given, 0), cap);
  const int first = a.start != nullptr ? after_wait(a.start)[s] : 0, start = min(max(first, 0), len);
  const int listed = after_wait(a.n_keep)[s];
  const int n = min(min(max(listed, 0), a.keep_cols), min(len, out_cap) - min(start, out_cap));
  if (head && tid == 0) {
    a.lens_out[s] = start + n;
    if (given > cap || first > len || listed > n) atomicOr(a.status, kStatusBadIndex);
  }
  const int32_t* keep = after_wait(a.keep) + static_cast<size_t>(s) * a.keep_cols;
  const int32_t* from_row = after_wait(a.table) + static_cast<size_t>(s) * a.cols;
  const int32_t* to_row = after_wait(a.table_out) + static_cast<size_t>(s) * a.out_cols;
  const int mask = (1 << a.page_shift) - 1, page_vecs = a.row_vecs << a.page_shift;
  uint4* pool = static_cast<uint4*>(pools.p[blockIdx.y]) + static_cast<size_t>(h) * page_vecs;
  const size_t page_stride = static_cast<size_t>(a.Hkv) * page_vecs;
  const int vec = tid % a.row_vecs, at = tid / a.row_vecs, step = kCompactThreads / a.row_vecs;
  for (int j0 = 0; j0 < n; j0 += step * kCompactUnroll) {
    uint4 x[kCompactUnroll];
    long long to[kCompactUnroll];
#pragma unroll
    for (int k = 0; k < kCompactUnroll; ++k) {
      const int j = j0 + k * step + at;
      to[k] = -1;
      if (j >= n) continue;
      const int e = keep[j], d = start + j;
      bool ok = e >= d && e < len && (j == 0 || keep[j - 1] < e);
      const int p = ok ? from_row[e >> a.page_shift] : -1, q = to_row[d >> a.page_shift];
      ok = p >= 0 && p < a.n_pages && q >= 0 && q < a.n_pages;
      const bool stays = p == q && e == d;
      if (ok && !stays && a.refs != nullptr) ok = after_wait(a.refs)[q] == 1;  // no other sequence's page
      if (!ok && head && vec == 0) atomicOr(a.status, kStatusBadIndex);
      if (!ok || stays) continue;
      x[k] = pool[p * page_stride + (e & mask) * a.row_vecs + vec];
      to[k] = static_cast<long long>(q * page_stride + (d & mask) * a.row_vecs + vec);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kCompactUnroll; ++k)
      if (to[k] >= 0) pool[to[k]] = x[k];
  }
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

cudaError_t launch_paged_compact(const CompactArgs& a, const PoolList& pools, cudaStream_t s) {
  ZSAA_LAUNCH(compact_kernel, dim3(a.S, pools.n, a.Hkv), dim3(kCompactThreads), 0, s, a, pools);
  return cudaSuccess;
}

}  // namespace zsaa
