// Pages counted by reference: tables that grow and shrink (resize), sequences that continue
// others (fork), and entries moved together (compact).
//
// refs[page] counts the table entries that name a page; a page with none is free, and there is
// no other list of free pages.  A call that needs pages takes those of the lowest numbers, in
// the order of its rows and columns: what it takes follows from the counts alone, not from
// timing, although the counts themselves change by atomics (whose order does not matter).
//
// Bound by chains of round trips to L2 where little moves (64 sequences that grow by a few tokens: 5.9
// us on the GPU, lengths -> pages -> counts -> free pages -> places), by HBM where entries do (8
// sequences' caches in 32 layers pruned to half: 248 us, 6.6 TB/s).
#include <algorithm>

#include "common.cuh"
#include "paged.h"

namespace zsaa {
namespace {

// As launch_kernel, in clusters of `ctas` along x.
template <typename... KArgs, typename... Args>
cudaError_t launch_cluster(void (*kernel)(KArgs...), dim3 grid, dim3 block, int ctas, size_t smem, cudaStream_t s,
                           Args&&... args) {
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

// One cluster, or one CTA where there is little, does a call: its CTAs change the counts, meet,
// count the free pages of their blocks of the pool, exchange the counts, and hand out the pages.  (No
// count outlives the call, so a pool's state is refs alone and a call needs no workspace.)  512
// sequences that come and go over 131072 pages: 12.5 us with blocks of 256 pages dealt out
// to the warps; 15.5 with one contiguous part of the pool to a CTA, because the pages that
// are taken lie in the lowest part; 28 with the counts changed by the cluster alone and a search for
// each page's row.
constexpr int kTakeThreads = 1024, kTakeWarps = kTakeThreads / 32, kTakeCtas = 8;
constexpr int kTakeBlock = 128;    // columns of a table row that a warp looks at together
constexpr int kTakeMasks = 32;     // words of free pages that a warp keeps
constexpr int kTakeFew = 16384;    // pages that one CTA looks through
constexpr int kTakeBlocks = 2048;  // blocks of a pool, at most

// A pool in blocks of 256 pages, or larger ones where there would be too many.
__host__ __device__ inline int block_shift(int n_pages) {
  int shift = 8;
  while (n_pages > (kTakeBlocks << shift)) ++shift;
  return shift;
}

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

__device__ __forceinline__ int running_sum(int v) {  // over the warp's lanes, own one included
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += x;
  }
  return v;
}
// the sum of the warps before this one, and of all (32 warps)
__device__ __forceinline__ int before_warp(const int* of_warp, int& total) {
  const int lane = threadIdx.x & 31, mine = of_warp[lane], run = running_sum(mine);
  total = __shfl_sync(0xffffffffu, run, 31);
  return __shfl_sync(0xffffffffu, run - mine, threadIdx.x >> 5);
}
__device__ __forceinline__ void meet(int ctas) {
  if (ctas > 1) cluster_sync_all(); else __syncthreads();
}

// The row of place k, at or behind row `lo`: the last with base[row] <= k (a whole warp).
__device__ __forceinline__ int row_of_place(const int* base, int lo, int rows, int k) {
  const int lane = threadIdx.x & 31;
  int n = rows - lo;
  while (n > 1) {
    const int step = (n + 31) >> 5, i = lane * step;
    const int at = (__popc(__ballot_sync(0xffffffffu, i < n && base[lo + i] <= k)) - 1) * step;
    lo += at;
    n = min(step, n - at);
  }
  return lo;
}

// Warp gw of `warps` gives up or shares its part of the rows' pages, each row's columns
// [touch(i), end(i)).
template <bool FORK, typename Touch>
__device__ __forceinline__ void touch_pages(const PagesArgs& a, int gw, int warps, Touch&& columns) {
  const int lane = threadIdx.x & 31, blocks = (a.cols + kTakeBlock - 1) / kTakeBlock;
  const unsigned units = static_cast<unsigned>(a.rows) * blocks;  // (a table has fewer than 2^31 entries)
#pragma unroll 2
  for (unsigned u = gw; u < units; u += warps) {
    const int i = static_cast<int>(u / static_cast<unsigned>(blocks));
    const int c0 = static_cast<int>(u - i * static_cast<unsigned>(blocks)) * kTakeBlock;
    const int2 t = columns(i);
    if (t.x >= c0 + kTakeBlock || t.y <= c0) continue;
    const int32_t* row = a.table + static_cast<size_t>(FORK ? a.parent[i] : i) * a.cols;
    int page[kTakeBlock / 32];
#pragma unroll
    for (int k = 0; k < kTakeBlock / 32; ++k) {
      const int c = c0 + 32 * k + lane;
      page[k] = c >= t.x && c < t.y ? row[c] : -1;
    }
#pragma unroll
    for (int k = 0; k < kTakeBlock / 32; ++k) {
      const int c = c0 + 32 * k + lane;
      if (c < t.x || c >= t.y) continue;
      if (FORK) a.table_out[static_cast<size_t>(i) * a.cols + c] = page[k];
      if (page[k] < 0 || page[k] >= a.n_pages) atomicOr(a.status, kStatusBadIndex);
      else atomicAdd(a.refs + page[k], FORK ? 1 : -1);
    }
  }
}

template <bool FORK>
__device__ __forceinline__ PagesArgs args_after_wait(const PagesArgs& given) {
  PagesArgs a = given;
  a.refs = after_wait(a.refs), a.table = after_wait(a.table), a.lens = after_wait(a.lens);
  if (FORK) a.parent = after_wait(a.parent), a.at = after_wait(a.at);
  else a.want = after_wait(a.want);
  return a;
}

// The pages given up or shared, on the whole device (calls that touch many: 32000 in 4 us).
template <bool FORK>
__global__ void __launch_bounds__(256) pages_touch_kernel(const __grid_constant__ PagesArgs given) {
  pdl_trigger();
  pdl_wait();
  const PagesArgs a = args_after_wait<FORK>(given);
  touch_pages<FORK>(a, static_cast<int>(blockIdx.x * 8 + (threadIdx.x >> 5)), static_cast<int>(gridDim.x) * 8, [&](int i) {
    const TakeRow r = take_row<FORK>(a, i);
    return make_int2(r.touch0, r.touch1);
  });
}

template <bool FORK>
__global__ void __launch_bounds__(kTakeThreads, 1) pages_take_kernel(const __grid_constant__ PagesArgs given, bool touched) {
  extern __shared__ int dynamic[];
  __shared__ int warp_sum[kTakeWarps], in_block[kTakeBlocks];  // in_block: free pages of each block, then before it
  __shared__ unsigned char lists[kTakeWarps * 256];
  pdl_trigger();
  int* base = dynamic;                 // [rows + 1]: pages that earlier rows need
  int* touch = base + given.rows + 1;  // [rows]: first column given up or shared
  int* end = touch + given.rows;       // [rows]: the column behind the last; the first that gets a page
  unsigned* masks = reinterpret_cast<unsigned*>(end + given.rows);  // free pages of a warp's blocks, 32 to a word
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = static_cast<int>(cluster_rank()), ctas = static_cast<int>(cluster_size());
  const int gw = rank * kTakeWarps + warp, warps = ctas * kTakeWarps;
  pdl_wait();
  const PagesArgs a = args_after_wait<FORK>(given);

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
  const int run = running_sum(mine);
  if (lane == 31) warp_sum[warp] = run;
  __syncthreads();
  int total_need;
  int before = run - mine + before_warp(warp_sum, total_need);
  for (int i = i0; i < i1; ++i) {
    const int need = base[i];
    base[i] = before;
    before += need;
  }
  if (tid == 0) base[a.rows] = total_need;

  // pages given up or shared.  (A count that falls below 0 is found with the free pages.)
  if (!touched) {
    touch_pages<FORK>(a, gw, warps, [&](int i) { return make_int2(touch[i], end[i]); });
    if (ctas > 1) __threadfence();
  }
  meet(ctas);

  // The free pages, block by block of the pool.  The lowest are taken first, so the warps' blocks
  // alternate, and each CTA gets the counts of all.
  const int shift = block_shift(a.n_pages), block_words = 1 << (shift - 5), blocks = (a.n_pages + (1 << shift) - 1) >> shift;
  const int words = ((blocks + warps - 1) / warps) << (shift - 5);  // of a warp
  const bool kept = words <= kTakeMasks;
  auto block_of = [&](int w) { return (w >> (shift - 5)) * warps + gw; };  // of this warp's word w
  auto page_of = [&](int w) {                                              // its first page
    return (static_cast<long long>(block_of(w)) << shift) + 32 * (w & (block_words - 1));
  };
  auto count_at = [&](int w) {
    const long long q = page_of(w) + lane;
    return q < a.n_pages ? __ldcg(a.refs + q) : 1;
  };
  int n_free = 0;
  // (a block that the pool's end cuts is gone through to its own end: its last word stores its count)
  for (int w0 = 0; w0 < words && block_of(w0) < blocks; w0 += 16) {
    int c[16], least = 1;
    unsigned mine_mask = 0;  // lane k: word w0 + k
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if (w0 + k < words) c[k] = count_at(w0 + k);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      if (w0 + k >= words) break;
      const unsigned m = __ballot_sync(0xffffffffu, c[k] <= 0);
      least = min(least, c[k]);
      if (lane == k) mine_mask = m;
      n_free += __popc(m);
      if (((w0 + k + 1) & (block_words - 1)) == 0) {
        const int block = block_of(w0 + k);
        if (lane < ctas && block < blocks) st_cluster_u32(smem_u32(&in_block[block]), lane, n_free);
        n_free = 0;
      }
    }
    if (kept && lane < 16 && w0 + lane < words) masks[warp * words + w0 + lane] = mine_mask;
    if (least < 0) {  // more given up than there were
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (w0 + k < words && c[k] < 0) a.refs[page_of(w0 + k) + lane] = 0;
      atomicOr(a.status, kStatusBadIndex);
    }
  }
  meet(ctas);
  int free_total, free_before = 0;  // (of the warp's first block)
  if (blocks <= 32) {
    const int here = lane < blocks ? in_block[lane] : 0, sum = running_sum(here);
    free_total = __shfl_sync(0xffffffffu, sum, 31);
    free_before = __shfl_sync(0xffffffffu, sum - here, gw & 31);
  } else {
    constexpr int PER = kTakeBlocks / kTakeThreads;
    int of_block[PER], here = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      of_block[i] = tid * PER + i < blocks ? in_block[tid * PER + i] : 0;
      here += of_block[i];
    }
    const int sum = running_sum(here);
    if (lane == 31) warp_sum[warp] = sum;
    __syncthreads();
    int at = sum - here + before_warp(warp_sum, free_total);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (tid * PER + i < blocks) in_block[tid * PER + i] = at;
      at += of_block[i];
    }
    __syncthreads();
    if (gw < blocks) free_before = in_block[gw];
  }

  // The free page of rank k goes to the k-th place that needs one.  A warp lists the free ones of
  // 256 pages, so that its lanes then have neighbouring places, which mostly are in one row: the
  // rows of the first and the last are looked for by the whole warp.
  unsigned char* list = lists + warp * 256;
  int lo = -1;
  for (int w0 = 0; w0 < words && page_of(w0) < a.n_pages; w0 += 8) {
    if (w0 > 0 && (w0 & (block_words - 1)) == 0) free_before = in_block[block_of(w0)];
    if (free_before >= total_need) break;
    const int q0 = static_cast<int>(page_of(w0));
    int n = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const unsigned mask = kept ? masks[warp * words + w0 + w] : __ballot_sync(0xffffffffu, count_at(w0 + w) <= 0);
      if (mask >> lane & 1) list[n + __popc(mask & ((1u << lane) - 1))] = static_cast<unsigned char>(32 * w + lane);
      n += __popc(mask);
    }
    __syncwarp();
    const int wanted = min(n, total_need - free_before);
    for (int i = 0; i < wanted; i += 32) {
      const int first = free_before + i, k = first + lane, last = min(first + 32, free_before + wanted) - 1;
      if (lo < 0 || base[lo + 1] <= first) lo = row_of_place(base, max(lo, 0), a.rows, first);
      const int hi = base[lo + 1] > last ? lo : row_of_place(base, lo, a.rows, last);
      if (k <= last) {
        int row = lo, m = hi - lo + 1;  // base[row] <= k < base[row + m]
        while (m > 1) {
          const int half = m >> 1;
          if (base[row + half] <= k) row += half, m -= half; else m = half;
        }
        const int page = q0 + list[i + lane];
        a.table_out[static_cast<size_t>(row) * a.cols + end[row] + (k - base[row])] = page;
        a.refs[page] = 1;
      }
      lo = hi;
    }
    free_before += n;
    __syncwarp();  // (the list is written again)
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
  const long long units = static_cast<long long>(a.rows) * ((a.cols + kTakeBlock - 1) / kTakeBlock);
  const int ctas = a.n_pages > kTakeFew || units > 2 * kTakeWarps ? kTakeCtas : 1;
  const bool many = units > kTakeCtas * kTakeWarps;
  const int shift = block_shift(a.n_pages), blocks = (a.n_pages + (1 << shift) - 1) >> shift;
  const int words = ((blocks + ctas * kTakeWarps - 1) / (ctas * kTakeWarps)) << (shift - 5);
  const size_t smem = sizeof(int) * (3 * static_cast<size_t>(a.rows) + 1 + (words <= kTakeMasks ? words * kTakeWarps : 0));
  static OncePerDevice once;
  const cudaError_t e = set_smem_limit_once(once, pages_take_kernel<FORK>,
                                            static_cast<int>(sizeof(int)) * (3 * kPagesMaxRows + 1 + kTakeMasks * kTakeWarps));
  if (e != cudaSuccess) return e;
  const dim3 touch(static_cast<unsigned>(std::min((units + 7) / 8, 1024ll)));
  if (many) ZSAA_LAUNCH(pages_touch_kernel<FORK>, touch, dim3(256), 0, s, a);
  return launch_cluster(pages_take_kernel<FORK>, dim3(ctas), dim3(kTakeThreads), ctas, smem, s, a, many);
}

// ---------------------------------------------------------------- fork: the partly filled pages

// One child and pool per CTA.  128 children of 16 sequences in 32 layers: 0.58 GB written, as much
// read (mostly from L2), in 148 us.

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
  const int all = n * a.Hkv;
#pragma unroll 4
  for (int v = tid; v < all; v += blockDim.x) {
    const int h = v / n;
    const size_t at = static_cast<size_t>(h) * stride + (v - h * n);
    d[at] = s[at];
  }
}

// ---------------------------------------------------------------- compact

// A cluster of CTAs (often one) moves some heads' entries of one sequence in one pool, a tile of
// entries after the other: the tile's loads, a barrier of the cluster, its stores.  Entry start + j
// comes from keep[j] >= start + j, so what a tile writes is never read by a later one, and in
// place is as right as into other pages.  While a tile's values are on their way the next tile's
// places are looked up (keep -> table -> page, three round trips), so a tile costs about one
// round trip.
//
// Moved into other pages no tile waits for another, and clusters as many as run at once share a list:
// 16250 of 65000 entries of one layer 26 us (5.1 TB/s), where one cluster to a head takes 34 and a CTA
// to a head 675.  (Two tiles on their way with the cluster's barrier split around the second's loads:
// 43 against 39 for the cluster's form.)  Three CTAs to an SM leave 80 registers a thread: 8 bytes spill.
constexpr int kCompactPerSm = 3;
constexpr int kCompactThreads = 256, kCompactUnroll = 8, kCompactVecs = kCompactThreads * kCompactUnroll;

struct CompactPlan {
  int heads;   // of a CTA
  int slices;  // CTAs of a head, each with a part of its dims (heads is 1 then)
  int vecs;    // 16-byte vectors of a CTA's part of an entry: a power of two, 8 or more
  int tile;    // entries of a CTA's share of a tile: heads * tile * vecs <= kCompactVecs
  int ctas;    // of a cluster
  int clusters;
};

__global__ void __launch_bounds__(kCompactThreads, kCompactPerSm)
    compact_kernel(const __grid_constant__ CompactArgs a, const __grid_constant__ PoolList pools,
                   const __grid_constant__ CompactPlan plan) {
  __shared__ int s_from[2][kCompactThreads], s_to[2][kCompactThreads];  // entries in the pool (of head 0), or -1
  pdl_trigger();
  pdl_wait();
  const int shares = plan.ctas * plan.clusters, s = static_cast<int>(blockIdx.x) / shares, tid = threadIdx.x;
  const int rank = static_cast<int>(blockIdx.x) - s * shares;
  const int part = static_cast<int>(blockIdx.z) / plan.slices, slice = static_cast<int>(blockIdx.z) - part * plan.slices;
  const int h0 = part * plan.heads, heads = min(plan.heads, a.Hkv - h0);
  const bool first_cta = blockIdx.y == 0 && blockIdx.z == 0;
  const int given = after_wait(a.lens)[s], cap = a.cols << a.page_shift, out_cap = a.out_cols << a.page_shift;
  const int len = min(max(given, 0), cap);
  const int begin = a.start != nullptr ? after_wait(a.start)[s] : 0, start = min(max(begin, 0), len);
  const int listed = after_wait(a.n_keep)[s];
  const int n = min(min(max(listed, 0), a.keep_cols), min(len, out_cap) - min(start, out_cap));
  if (first_cta && rank == 0 && tid == 0) {
    a.lens_out[s] = min(start, out_cap) + n;
    if (given > cap || begin > len || start > out_cap || listed > n) atomicOr(a.status, kStatusBadIndex);
  }
  const int32_t* keep = after_wait(a.keep) + static_cast<size_t>(s) * a.keep_cols;
  const int32_t* from_row = after_wait(a.table) + static_cast<size_t>(s) * a.cols;
  const int32_t* to_row = after_wait(a.table_out) + static_cast<size_t>(s) * a.out_cols;
  const int mask = (1 << a.page_shift) - 1;
  // Where no page is both read and written all shares go at once, each for itself; else one
  // cluster's do, tile by tile.
  bool in_place = a.table_out == a.table;
  if (!in_place) {
    bool same = false;
    for (int c = (start >> a.page_shift) + tid; n > 0 && c <= (start + n - 1) >> a.page_shift; c += kCompactThreads)
      same |= c < a.cols && to_row[c] == from_row[c];
    in_place = __syncthreads_or(same) != 0;
  }
  if (in_place && rank >= plan.ctas) return;  // (whole clusters)
  const unsigned step = plan.tile * (in_place ? plan.ctas : shares), end = n;
  // thread i < tile looks entry i of this CTA's share up: first its list entry, a tile later its pages
  const unsigned mine = rank * plan.tile + tid;
  int e = -1, before = -1;
  auto look = [&](unsigned j0) {  // (j0 may pass 2^31)
    const unsigned j = j0 + mine;
    if (tid < plan.tile && j < end) {
      e = keep[j];
      before = j > 0 ? keep[j - 1] : -1;
    }
  };
  auto place = [&](unsigned j0, int slot) {
    const unsigned j = j0 + mine;
    if (tid >= plan.tile) return;
    int from = -1, to = -1;
    if (j < end) {
      const int d = start + static_cast<int>(j), q = to_row[d >> a.page_shift];
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
    s_from[slot][tid] = from;
    s_to[slot][tid] = to;
  };
  const int row_shift = 31 - __clz(a.row_vecs), part_shift = 31 - __clz(plan.vecs);
  uint4* pool = static_cast<uint4*>(pools.p[blockIdx.y]) + slice * plan.vecs + (tid & (plan.vecs - 1));
  const int at = tid >> part_shift, rows = kCompactThreads >> part_shift;  // (head, entry) pairs of a round
  look(0);
  place(0, 0);
  look(step);
  __syncthreads();
  int slot = 0;
  for (unsigned j0 = 0; j0 < end; j0 += step, slot ^= 1) {
    uint4 x[kCompactUnroll];
    int to[kCompactUnroll];
#pragma unroll
    for (int k = 0; k < kCompactUnroll; ++k) {
      const int i = k * rows + at, h = i / plan.tile, r = i - h * plan.tile;
      to[k] = -1;
      if (h >= heads) continue;
      const int from = s_from[slot][r], head = (h0 + h) << a.page_shift;
      if (from < 0) continue;
      x[k] = pool[static_cast<size_t>(from + head) << row_shift];
      to[k] = s_to[slot][r] + head;
    }
    place(j0 + step, slot ^ 1);
    look(j0 + 2 * step);
    if (in_place && plan.ctas > 1) cluster_sync_all(); else __syncthreads();
#pragma unroll
    for (int k = 0; k < kCompactUnroll; ++k)
      if (to[k] >= 0) pool[static_cast<size_t>(to[k]) << row_shift] = x[k];
  }
}

// A CTA takes as many heads as its registers hold of the longest list.  Where the CTAs would not
// fill the SMs the list is split over a cluster; a move in place splits a head's dims first (down to
// 128 bytes), one into another table takes as many clusters as run at once.
CompactPlan compact_plan(const CompactArgs& a, int pools, int sms) {
  CompactPlan p{1, 1, a.row_vecs, 0, 1, 1};
  const bool in_place = a.table_out == a.table;
  p.heads = std::max(1, std::min(a.Hkv, kCompactVecs / (a.row_vecs * std::min(a.keep_cols, kCompactVecs / a.row_vecs))));
  const long long ctas = static_cast<long long>(a.S) * pools * ((a.Hkv + p.heads - 1) / p.heads);
  while (in_place && p.heads == 1 && p.vecs > 8 && ctas * p.slices < 2 * sms) p.slices *= 2, p.vecs /= 2;
  p.tile = std::min(kCompactVecs / (p.heads * p.vecs), a.keep_cols);
  while (p.ctas < 8 && ctas * p.slices * p.ctas < 2 * sms && p.tile * p.ctas < a.keep_cols) p.ctas *= 2;
  if (!in_place && p.ctas == 8) {
    const long long at_once = kCompactPerSm * sms / (8 * ctas), tiles = (a.keep_cols + 8ll * p.tile - 1) / (8 * p.tile);
    p.clusters = static_cast<int>(std::max(1ll, std::min(at_once, tiles)));
  }
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
  const dim3 grid(a.S * p.ctas * p.clusters, pools.n, (a.Hkv + p.heads - 1) / p.heads * p.slices);
  return launch_cluster(compact_kernel, grid, dim3(kCompactThreads), p.ctas, 0, s, a, pools, p);
}

}  // namespace zsaa
