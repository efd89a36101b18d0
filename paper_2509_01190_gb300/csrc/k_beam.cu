// Beam search over a batch: selection of the best continuations, and page tables
// that follow the selected beams.
//
// Selection.  Beam w of a batch element has a running score s_w and logits x_w over
// V tokens; continuation (w, v) has the total s_w + x_w[v] - lse(x_w), lse(x) =
// log sum exp(x).  The K largest totals are wanted; lse moves a whole beam, so a
// beam's own order is that of its logits and one pass over them is enough:
//   beam_scan_kernel   one stretch of one beam's logits per CTA: its sum of exponentials
//                      and its K best tokens, in order;
//   beam_merge_kernel  one CTA per batch element: every beam's lse and K best tokens
//                      from its stretches', then the K best totals of all beams.
// The logits are read once, which bounds large batches; few beams are bound by the
// two kernels' own chains.
//
// The K best without a sort and without a list while the logits pass: a thread keeps the
// maximum of its values alone.  Every warp then publishes the best of its lanes' maxima,
// at least K in all; the K-th best published value is a lower bound of the K-th best of
// all, so only the threads whose maximum reaches it look at their values again (in L2),
// and the few values that do are ranked by counting.  Values are compared together with
// their place, lower place first; where the bound is the stretch's minimum (a banned
// vocabulary, whatever number marks it; a NaN counts as -inf) the first 2 K places hold the
// K best or more, and where more values than the list holds reach the bound all the same,
// the K-th best is found bit by bit instead.
//
// Sums are taken against a logit: a warp's against the maximum of its first values, brought
// to its last maximum at the end; warps and stretches are put together against the larger of
// their maxima, by the factor exp(their own - the larger).  A reference that is itself a
// float32 logit makes x - reference exact where it matters, next to the maximum, at every
// size of the logits, and a maximum's own term 1.  (Differences are taken before the product
// with log2(e): the other way around a logit of 1000 would be off by 1e-4.)  A thread's
// terms are added in 32 bits and everything after that as 64-bit integers of 2^-36: FP64
// runs at a sixty-fourth of FP32 here, and is left to a beam's logarithm and the totals of
// its K tokens.
#include <algorithm>

#include "common.cuh"
#include "paged.cuh"

namespace zsaa {
namespace {

constexpr int kScanWarps = 8, kScanThreads = 32 * kScanWarps;
constexpr int kScanGroups = 4;                              // 16-byte loads of a thread in a step
constexpr int kScanTile = 4 * kScanGroups * kScanThreads;  // values of a CTA's step
constexpr int kPublish = 8;                                 // lane maxima that a warp publishes, at most
constexpr int kListCap = 512;                               // collected values, at most
constexpr int kMergeThreads = 512;
constexpr int kMergeWarps = kMergeThreads / 32;
constexpr int kMergeDepth = 8;  // elements of each list that the merge holds in shared memory
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSumUnit = 0x1p36f;  // (2^26 terms of up to 1 fit)

// Order-preserving map of a float (no NaN) to unsigned; -0 equals +0, -inf is 0x007fffff.
__device__ __forceinline__ uint32_t float_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_float(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
// The same for a double; NaN is 0, below everything.
__device__ __forceinline__ uint64_t double_key(double x) {
  if (x != x) return 0;
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(x + 0.0));
  return u ^ (static_cast<uint64_t>(static_cast<int64_t>(u) >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ float key_double_to_float(uint64_t k) {
  if (k == 0) return __uint_as_float(0x7fffffffu);
  return static_cast<float>(__longlong_as_double(
      static_cast<long long>(k & 0x8000000000000000ull ? k ^ 0x8000000000000000ull : ~k)));
}

__device__ __forceinline__ uint64_t warp_max_u64(uint64_t v) {
  const uint32_t hi = static_cast<uint32_t>(v >> 32);
  const uint32_t top = __reduce_max_sync(0xffffffffu, hi);
  const uint32_t lo = __reduce_max_sync(0xffffffffu, hi == top ? static_cast<uint32_t>(v) : 0u);
  return static_cast<uint64_t>(top) << 32 | lo;
}

// maximum of three that is NaN where one of them is; minimum of three
__device__ __forceinline__ float fmax3_nan(float a, float b, float c) {
  float y;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ float fmin3(float a, float b, float c) {
  float y;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

// A value (no NaN) at a place: the higher value, then the lower place, is the larger.
__device__ __forceinline__ uint64_t value_at(float x, int place) {
  return static_cast<uint64_t>(float_key(x)) << 32 | static_cast<uint32_t>(~place);
}

// A sum against the maximum `own` as one against `top`, which is as large or larger; below
// e^-64 nothing of 2^62 is left.  (NaN, of two maxima of -inf, whose sums are 0: 0.)
__device__ __forceinline__ uint64_t sum_against(uint64_t sum, float own, float top) {
  const float d = own - top;
  if (d == 0.f) return sum;
  return d > -64.f ? __float2ull_rn(__ull2float_rn(sum) * expf(d)) : 0;
}

// One stretch: `tiles` steps of 4096 values.  A value's place is its token; a collected
// value is (key << 32 | ~token), so that a larger one is a better one.  NaN logits are
// ordered as -inf (their row's totals are all NaN).  Places before the row or past its end
// hold -inf and come after every real one: as unsigned, their ~token is smaller.
// Bound by its loads on large batches, and then by the end of the stretches: 192 beams of
// 128256 logits in 25 us from HBM, 3.9 TB/s, 58% of the copy rate (29 with a bound and a list kept
// up from step to step, whose barriers and rare branches then were most of the time).
__global__ void __launch_bounds__(kScanThreads, 4)
    beam_scan_kernel(const float* __restrict__ logits, long long ld, int V, int K, int chunks, int tiles,
                     const uint8_t* __restrict__ done, BeamChunk* __restrict__ stat, uint2* __restrict__ cand) {
  constexpr int GROUPS = kScanGroups, STEP = 4 * kScanThreads;
  __shared__ __align__(16) uint64_t pub[kScanWarps * kPublish];
  __shared__ uint64_t list[kListCap], s_bound, s_sum[kScanWarps];
  __shared__ int s_count, s_bad[kScanWarps], s_n[kScanWarps];
  __shared__ uint32_t s_least[kScanWarps];
  __shared__ float s_top[kScanWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = blockIdx.x / chunks, c = blockIdx.x % chunks;
  pdl_trigger();
  if (tid == 0) s_count = 0;
  pdl_wait();
  logits = after_wait(logits);
  done = after_wait(done);
  if (done != nullptr && done[row] != 0) return;  // its only continuation needs no logits
  const float* p = logits + static_cast<long long>(row) * ld;
  // 16-byte loads start up to 3 values before the row, at the boundary below it
  const int start = c * tiles * kScanTile - static_cast<int>((reinterpret_cast<uintptr_t>(p) >> 2) & 3);
  uint2* out = cand + static_cast<size_t>(blockIdx.x) * K;
  if (start >= V) {  // (only ever the row's last stretch)
    if (tid == 0) stat[blockIdx.x] = BeamChunk{0, -INFINITY, 0};
    for (int i = tid; i < K; i += kScanThreads) out[i] = make_uint2(0, 0);
    return;
  }
  const int n_tiles = min(tiles, (V - start + kScanTile - 1) / kScanTile);
  auto place = [&](int t, int i) { return start + t * kScanTile + i * STEP + tid * 4; };  // of a group's first value
  auto load = [&](int t, float4 (&f)[GROUPS]) {
    const int first = start + t * kScanTile;
    if (first >= 0 && first + kScanTile <= V) {
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) f[i] = __ldg(reinterpret_cast<const float4*>(p + place(t, i)));
      return;
    }
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const int u = place(t, i);
      f[i] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      if (u >= 0 && u <= V - 4) {
        f[i] = __ldg(reinterpret_cast<const float4*>(p + u));
      } else {
        if (u >= 0 && u < V) f[i].x = p[u];
        if (u + 1 >= 0 && u + 1 < V) f[i].y = p[u + 1];
        if (u + 2 >= 0 && u + 2 < V) f[i].z = p[u + 2];
        if (u + 3 >= 0 && u + 3 < V) f[i].w = p[u + 3];
      }
    }
  };
  auto max_of = [](const float4& f, float m) { return fmax3_nan(fmax3_nan(f.x, f.y, f.z), f.w, m); };

  float best = -INFINITY, least = INFINITY, first = -INFINITY, ref = 0.f;
  float s4[4] = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](const float4& f) {
    s4[0] += ex2_fast((f.x - ref) * kLog2e);
    s4[1] += ex2_fast((f.y - ref) * kLog2e);
    s4[2] += ex2_fast((f.z - ref) * kLog2e);
    s4[3] += ex2_fast((f.w - ref) * kLog2e);
  };
  float4 f[GROUPS];
  load(0, f);
  for (int t = 0; t < n_tiles; ++t) {
    float4 next[GROUPS];
    if (t + 1 < n_tiles) load(t + 1, next);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      best = max_of(f[i], best);
      least = fmin3(fmin3(f[i].x, f[i].y, f[i].z), f[i].w, least);
    }
    if (first == -INFINITY) {  // (warp-uniform) the reference: the first finite maximum
      first = key_float(__reduce_max_sync(0xffffffffu, float_key(fmaxf(best, -INFINITY))));
      ref = first == -INFINITY ? 0.f : first;
    }
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      add(f[i]);
      f[i] = next[i];
    }
  }
  // what few stretches need
  bool bad = !(best < INFINITY);
  if (bad) {  // a NaN or +inf: the maximum of the numbers; a NaN is a -inf among them
    best = -INFINITY;
    for (int t = 0; t < n_tiles; ++t) {
      load(t, f);
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        const float m = max_of(f[i], -INFINITY);
        if (m != m) least = -INFINITY;
        best = fmaxf(best, fmaxf(fmaxf(f[i].x, f[i].y), fmaxf(f[i].z, f[i].w)));
      }
    }
  }
  const float m = key_float(__reduce_max_sync(0xffffffffu, float_key(best)));
  if (m - ref > 40.f && first != -INFINITY) {  // (warp-uniform) the first values were far below: the sum again
    ref = m;
    s4[0] = s4[1] = s4[2] = s4[3] = 0.f;
    for (int t = 0; t < n_tiles; ++t) {
      load(t, f);
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) add(f[i]);
    }
  }
  // against the last maximum, as integers
  bad = __any_sync(0xffffffffu, bad);
  const float step = m > ref ? expf(ref - m) : 1.f;  // (e^-40 or more, but for a maximum of +inf)
  uint64_t sum = __float2ull_rn(((s4[0] + s4[1]) + (s4[2] + s4[3])) * step * kSumUnit);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  // the bound: in place of its own place a maximum has the thread's last one
  uint64_t mine = value_at(best, place(n_tiles - 1, GROUPS - 1) + 3);
  const int publish = min(kPublish, 2 * ((K + kScanWarps - 1) / kScanWarps));  // twice what K needs, for a closer bound
  for (int k = 0; k < publish; ++k) {
    const uint64_t x = warp_max_u64(mine);
    if (lane == 0) pub[warp * publish + k] = x;
    if (mine == x) mine = 0;
  }
  const uint32_t low = __reduce_min_sync(0xffffffffu, float_key(least));
  if (lane == 0) {
    s_sum[warp] = sum;
    s_top[warp] = m;
    s_bad[warp] = bad;
    s_least[warp] = low;
  }
  __syncthreads();
  if (tid < kScanWarps * publish) {
    const uint64_t x = pub[tid];
    int r = 0;
    for (int j = 0; j < kScanWarps * publish; j += 8) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(pub + j + i);
        r += (y.x > x) + (y.y > x);
      }
    }
    if (r == K - 1) s_bound = x;
  }
  __syncthreads();
  uint64_t bound = s_bound;
  uint32_t lowest = s_least[0];
#pragma unroll
  for (int w = 1; w < kScanWarps; ++w) lowest = min(lowest, s_least[w]);
  if (static_cast<uint32_t>(bound >> 32) == lowest)
    bound = static_cast<uint64_t>(lowest) << 32 | static_cast<uint32_t>(~(max(start, 0) + 2 * K - 1));
  // The values of the threads whose maximum, at its first place, reaches the bound: the
  // whole warp looks at them, a group a lane, in a round trip or two.
  auto collect = [&](uint64_t from) {
    const unsigned todo = __ballot_sync(0xffffffffu, value_at(best, max(place(0, 0), 0)) >= from);
    const unsigned per = n_tiles * GROUPS, all = __popc(todo) * per;
    for (unsigned e = lane; e < all; e += 32) {
      const unsigned k = e / per, g = e - k * per;  // the k-th of those threads, its group
      unsigned t = todo;
      for (unsigned i = 0; i < k; ++i) t &= t - 1;
      const int u = start + (warp * 32 + __ffs(t) - 1) * 4 + static_cast<int>(g / GROUPS * kScanTile + g % GROUPS * STEP);
      float v[4];
      if (u >= 0 && u <= V - 4) {
        const float4 x = __ldg(reinterpret_cast<const float4*>(p + u));
        v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = u + j >= 0 && u + j < V ? p[u + j] : -INFINITY;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t x = value_at(fmaxf(v[j], -INFINITY), u + j);
        if (x >= from) {
          const int n = atomicAdd(&s_count, 1);
          if (n < kListCap) list[n] = x;
        }
      }
    }
  };
  collect(bound);
  __syncthreads();
  int n = s_count;
  if (n > kListCap) {  // block-uniform: the K-th largest value, bit by bit
    bound = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t from = bound | (1ull << bit);
      int have = 0;
      if (value_at(best, max(place(0, 0), 0)) >= from)
        for (int t = 0; t < n_tiles; ++t) {
          load(t, f);
#pragma unroll
          for (int i = 0; i < GROUPS; ++i) {
            const int u = place(t, i);
            have += (value_at(fmaxf(f[i].x, -INFINITY), u) >= from) + (value_at(fmaxf(f[i].y, -INFINITY), u + 1) >= from) +
                    (value_at(fmaxf(f[i].z, -INFINITY), u + 2) >= from) + (value_at(fmaxf(f[i].w, -INFINITY), u + 3) >= from);
          }
        }
      have = __reduce_add_sync(0xffffffffu, have);
      __syncthreads();  // the previous round's counts are read
      if (lane == 0) s_n[warp] = have;
      __syncthreads();
      int all = 0;
      for (int w = 0; w < kScanWarps; ++w) all += s_n[w];
      if (all >= K) bound = from;
    }
    __syncthreads();
    if (tid == 0) s_count = 0;
    __syncthreads();
    collect(bound);
    __syncthreads();
    n = s_count;
  }
  if (warp == kScanWarps - 1) {  // (few lists reach this warp) the warps' sums, one a lane
    const bool in = lane < kScanWarps;
    const float own = in ? s_top[lane] : -INFINITY, top = warp_max(own);
    const bool any_bad = __any_sync(0xffffffffu, in && s_bad[lane] != 0);
    uint64_t x = in ? sum_against(s_sum[lane], own, top) : 0;
#pragma unroll
    for (int o = kScanWarps / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (lane == 0) stat[blockIdx.x] = BeamChunk{x, top, any_bad};
  }
  for (int i = tid; i < n; i += kScanThreads) {  // (at least K: a step has more places than that)
    const uint64_t x = list[i];
    int r = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) r += list[j] > x;
    const uint32_t token = ~static_cast<uint32_t>(x);
    if (r < K) out[r] = token < static_cast<uint32_t>(V) ? make_uint2(static_cast<uint32_t>(x >> 32), token) : make_uint2(0, 0);
  }
}

// Half of the warps put the beams' sums together, the other half their lists; what more than
// kSumWarps beams have, all of them.
constexpr int kSumWarps = kMergeWarps / 2;

// An element and another beam: up to so many such pairs are ranked by counting, more take a
// merge of the beams' lists by one warp (us of 24 selections from 32000 logits a beam, counting
// and merge: 8 beams with 8 tokens, 512 pairs, 12.0 and 12.9; with 16, 1024, 15.8 and 17.6; 16
// beams with 16, 4096, 31.3 and 27.4).
constexpr int kRankPairs = 1024;

// 8 bytes from device memory to this thread's place in shared memory
__device__ __forceinline__ void cp_async8(void* to, const void* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}

// Bound by its chain of steps: 8 tokens of 8 beams 6 us, 64 of 64 beams 80 (cold).
__global__ void __launch_bounds__(kMergeThreads)
    beam_merge_kernel(const BeamChunk* __restrict__ stat, const uint2* __restrict__ cand, int W, int V, int K,
                      int chunks, const float* __restrict__ scores, const uint8_t* __restrict__ done, int eos,
                      float* __restrict__ scores_out, int32_t* __restrict__ parent, int32_t* __restrict__ token,
                      uint8_t* __restrict__ done_out) {
  extern __shared__ __align__(16) uint8_t smem[];
  const int list_warps = W > kSumWarps ? kMergeWarps : kSumWarps;
  uint64_t* total = reinterpret_cast<uint64_t*>(smem);    // [W][K] ordered totals (0: none, or NaN)
  uint2* best = reinterpret_cast<uint2*>(total + W * K);  // [W][K] (key, token) in order; key 0: none
  uint2* merged = best + W * K;                           // [list warps][2][K] lists of the chunks merged so far
  uint2* cache = merged + list_warps * 2 * K;             // [list warps][depth][64] the lists' next elements
  __shared__ uint64_t s_sum[kBeamMaxBeams];
  __shared__ float s_top[kBeamMaxBeams];
  __shared__ double s_log[kBeamMaxBeams], s_score[kBeamMaxBeams];  // log of the sum against s_top
  __shared__ uint8_t s_done[kBeamMaxBeams], s_bad[kBeamMaxBeams];
  __shared__ int rank[kRankPairs];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.x, n = W * K;
  const bool few = n * W <= kRankPairs;
  pdl_trigger();
  pdl_wait();
  stat = after_wait(stat) + static_cast<size_t>(b) * W * chunks;
  cand = after_wait(cand) + static_cast<size_t>(b) * W * chunks * K;
  scores = after_wait(scores);
  done = after_wait(done);
  if (few)
    for (int i = tid; i < n; i += kMergeThreads) rank[i] = i % K;  // its place in its own beam's list
  // Beam w's best tokens in order.  The chunks' lists are in order: K times the best head of
  // two lists a lane, the list merged so far in place 0 and up to 63 chunks after it.  Equal
  // keys go by place, so the lower token comes first.  A list's next kMergeDepth elements
  // are in shared memory or on their way there, one asked for with each that is taken.
  auto merge_lists = [&](int w, int slot) {
    uint2* row = best + w * K;
    const uint2* lists = cand + static_cast<size_t>(w) * chunks * K;
    const uint2* so_far = nullptr;
    uint2* mine = cache + slot * kMergeDepth * 64 + lane;
    const bool over = done != nullptr && done[b * W + w] != 0;
    for (int c0 = 0; c0 < chunks; c0 += 63) {
      uint2* to = c0 + 63 >= chunks ? row : merged + (slot * 2 + (c0 / 63) % 2) * K;
      const uint2* at[2] = {nullptr, nullptr};
      int pos[2] = {0, 0};
      uint2 head[2];
      auto advance = [&](int i) {
        const int taken = pos[i]++;
        if (K <= kMergeDepth) {  // all there
          head[i] = pos[i] < K ? mine[pos[i] * 64 + 32 * i] : make_uint2(0, 0);
          return;
        }
        if (taken + kMergeDepth < K) cp_async8(&mine[taken % kMergeDepth * 64 + 32 * i], at[i] + taken + kMergeDepth);
        cp_async_commit();
        cp_async_wait<kMergeDepth - 1>();
        head[i] = pos[i] < K ? mine[pos[i] % kMergeDepth * 64 + 32 * i] : make_uint2(0, 0);
      };
#pragma unroll
      for (int i = 0; i < 2; ++i) {  // (all in flight together: one by one, each would cost its own round trip)
        const int c = c0 + lane + 32 * i - 1;
        at[i] = lane + 32 * i == 0 ? so_far : c < chunks ? lists + static_cast<size_t>(c) * K : nullptr;
        uint2 x[kMergeDepth];
#pragma unroll
        for (int k = 0; k < kMergeDepth; ++k) x[k] = at[i] != nullptr && k < K ? at[i][k] : make_uint2(0, 0);
#pragma unroll
        for (int k = 0; k < kMergeDepth; ++k) mine[k * 64 + 32 * i] = x[k];
        head[i] = x[0];
      }
      if (over) break;
      for (int k = 0; k < K; ++k) {
        const uint32_t x = __reduce_max_sync(0xffffffffu, max(head[0].x, head[1].x));
        const unsigned m0 = __ballot_sync(0xffffffffu, head[0].x == x), m1 = __ballot_sync(0xffffffffu, head[1].x == x);
        if (lane == __ffs(m0 != 0 ? m0 : m1) - 1) {
          if (m0 == 0) {
            to[k] = head[1];
            advance(1);
          } else if (lane > 0 || so_far == nullptr) {
            to[k] = head[0];
            if (at[0] != nullptr) advance(0);
          } else {  // (the list merged so far is in shared memory)
            to[k] = head[0];
            head[0] = ++pos[0] < K ? so_far[pos[0]] : make_uint2(0, 0);
          }
        }
      }
      cp_async_wait<0>();
      __syncwarp();
      so_far = to;
    }
    if (over)  // eos at no cost; the other tokens, in their order, are not allowed
      for (int k = lane; k < K; k += 32)
        row[k] = k >= V ? make_uint2(0, 0)
                        : make_uint2(k == 0 ? 0x80000000u : 0x007fffffu, k == 0 ? eos : k - 1 < eos ? k - 1 : k);
  };
  if (warp < kSumWarps) {
    for (int w = warp; w < W; w += kSumWarps) {
      // (every load of a beam in one round trip: what an ended one's are is of no account)
      const BeamChunk* st = stat + w * chunks;
      BeamChunk first = lane < chunks ? st[lane] : BeamChunk{0, -INFINITY, 0};
      const bool over = done != nullptr && done[b * W + w] != 0;
      const float score = scores == nullptr ? 0.f : scores[b * W + w];
      float top = first.top;
      int bad = first.bad;
      for (int c = lane + 32; c < chunks; c += 32) {
        const BeamChunk x = st[c];
        top = fmaxf(top, x.top);
        bad |= x.bad;
      }
      top = warp_max(top);
      bad = __any_sync(0xffffffffu, bad);
      uint64_t sum = sum_against(first.sum, first.top, top);
      for (int c = lane + 32; c < chunks; c += 32) sum += sum_against(st[c].sum, st[c].top, top);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (lane == 0) {
        s_sum[w] = sum;
        s_top[w] = top;
        s_bad[w] = bad;
        s_done[w] = over;
        s_score[w] = static_cast<double>(score);
      }
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kSumWarps * 32) : "memory");
    if (tid < W) {  // (a logarithm is a long chain of FP64: all beams' at once, while the lists are merged)
      double l;
      if (s_done[tid] || (!s_bad[tid] && s_top[tid] == -INFINITY)) {
        l = 0.0;  // eos at no cost; no allowed token: every total is -inf
        s_top[tid] = 0.f;
      } else if (s_bad[tid]) {
        l = __longlong_as_double(0x7ff8000000000000ll);  // every total NaN
      } else {
        l = log(static_cast<double>(s_sum[tid]) * (1.0 / kSumUnit));
      }
      s_log[tid] = l;
    }
    __syncwarp();
    for (int w = kSumWarps + warp; w < W; w += kMergeWarps) merge_lists(w, kSumWarps + warp);
  } else {
    for (int w = warp - kSumWarps; w < W; w += list_warps) merge_lists(w, warp - kSumWarps);
  }
  __syncthreads();
  for (int i = tid; i < n; i += kMergeThreads) {  // (the maximum off first: of floats, all but always exact)
    const double x = static_cast<double>(key_float(best[i].x)) - static_cast<double>(s_top[i / K]);
    total[i] = double_key(s_score[i / K] + (x - s_log[i / K]));
  }
  __syncthreads();
  auto put = [&](int r, int w, int i, uint64_t x) {  // total x of element i, beam w's, has rank r
    const size_t o = static_cast<size_t>(b) * K + r;
    const int tok = static_cast<int>(best[i].y);
    scores_out[o] = key_double_to_float(x);
    parent[o] = w;
    token[o] = tok;
    if (done_out != nullptr) done_out[o] = s_done[w] || tok == eos;
  };
  // A beam's totals fall along its list.  Few: an element's rank is the sum over the beams of
  // how many of theirs come before it (equal totals of an earlier beam do).
  if (few) {
    for (int e = tid; e < n * W; e += kMergeThreads) {
      const int i = e % n, u = e / n, w = i / K;
      if (u == w || best[i].x == 0) continue;
      const uint64_t x = total[i];
      int lo = 0, hi = K;  // the first element of beam u that does not come before
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        const uint64_t y = total[u * K + mid];
        if (best[u * K + mid].x != 0 && (y > x || (y == x && u < w))) lo = mid + 1; else hi = mid;
      }
      if (lo > 0) atomicAdd(&rank[i], lo);
    }
    __syncthreads();
    for (int i = tid; i < n; i += kMergeThreads)
      if (rank[i] < K && best[i].x != 0) put(rank[i], i / K, i, total[i]);
    return;
  }
  // Many: K times the best head of two beams a lane, equal totals by beam.
  if (warp > 0) return;
  uint64_t head[2];
  bool there[2];
  int pos[2] = {0, 0};
  auto look = [&](int i) {
    const int w = lane + 32 * i, at = w * K + pos[i];
    there[i] = w < W && pos[i] < K && best[at].x != 0;
    head[i] = there[i] ? total[at] : 0;
  };
  look(0);
  look(1);
  for (int r = 0; r < K; ++r) {
    const uint64_t x = warp_max_u64(max(head[0], head[1]));
    const unsigned m0 = __ballot_sync(0xffffffffu, there[0] && head[0] == x);
    const unsigned m1 = __ballot_sync(0xffffffffu, there[1] && head[1] == x);
    if (lane != __ffs(m0 != 0 ? m0 : m1) - 1) continue;
    const int i = m0 != 0 ? 0 : 1, w = lane + 32 * i;
    put(r, w, w * K + pos[i], x);
    if (i == 0) {
      ++pos[0];
      look(0);
    } else {
      ++pos[1];
      look(1);
    }
  }
}

// One CTA per (slot, layer's K or V).  Slot j of batch element b continues beam p =
// parent[b][j]: it takes over the parent's whole pages; the partly filled page stays
// with the parent's first child, and a later child gets its entries copied into its
// own fresh page.
struct ReorderArgs {
  PoolList pools;
  const int32_t *parent, *table, *lens, *fresh;
  int32_t *table_out, *lens_out;
  int W, K, cols, n_pages, page_shift, Hkv, row_vecs;  // row_vecs: 16-byte vectors of one entry of one head
  int* status;
};

__global__ void __launch_bounds__(256) beam_reorder_kernel(const __grid_constant__ ReorderArgs a) {
  pdl_trigger();
  pdl_wait();
  const int slot = blockIdx.x, b = slot / a.K, j = slot % a.K, tid = threadIdx.x;
  const int32_t* par = after_wait(a.parent) + static_cast<size_t>(b) * a.K;
  const int p = par[j];
  const bool head = blockIdx.y == 0;
  if (p < 0 || p >= a.W) {
    if (head && tid == 0) {
      a.lens_out[slot] = 0;
      atomicOr(a.status, kStatusBadIndex);
    }
    return;
  }
  const size_t src = static_cast<size_t>(b) * a.W + p;
  const int32_t* row = after_wait(a.table) + src * a.cols;
  const int cap = a.cols << a.page_shift;
  const int given = after_wait(a.lens)[src];
  const int len = min(max(given, 0), cap);
  const int whole = len >> a.page_shift, part = len & ((1 << a.page_shift) - 1);
  bool again = false;  // an earlier slot continues the same parent
  for (int i = tid; i < j; i += blockDim.x) again |= par[i] == p;
  again = __syncthreads_or(again) != 0;
  const bool own = part == 0 || again;  // the slot's next entries go to its fresh page
  const int to = after_wait(a.fresh)[slot];
  const bool copy = part != 0 && again;
  const int from = copy ? row[whole] : 0;
  const bool bad = given < 0 || given > cap || (own && whole < a.cols && (to < 0 || to >= a.n_pages)) ||
                   (copy && (from < 0 || from >= a.n_pages));
  if (head) {
    int32_t* out = a.table_out + static_cast<size_t>(slot) * a.cols;
    for (int i = tid; i < whole; i += blockDim.x) out[i] = row[i];
    if (tid == 0) {
      if (whole < a.cols) out[whole] = own ? to : row[whole];
      a.lens_out[slot] = len;
      if (bad) atomicOr(a.status, kStatusBadIndex);
    }
  }
  if (!copy || bad) return;
  const int n = part * a.row_vecs, stride = a.row_vecs << a.page_shift;  // vectors to copy, and of a page, per head
  uint4* pool = static_cast<uint4*>(a.pools.p[blockIdx.y]);
  const uint4* s = pool + static_cast<size_t>(from) * a.Hkv * stride;
  uint4* d = pool + static_cast<size_t>(to) * a.Hkv * stride;
  for (int h = 0; h < a.Hkv; ++h)
    for (int i = tid; i < n; i += blockDim.x) d[static_cast<size_t>(h) * stride + i] = s[static_cast<size_t>(h) * stride + i];
}

}  // namespace

int beam_chunks_most(int V) { return (V + 3 + kScanTile - 1) / kScanTile; }

cudaError_t launch_beam_select(const float* logits, long long ld, int B, int W, int V, const float* scores,
                               const uint8_t* done, int eos, int K, float* scores_out, int32_t* parent,
                               int32_t* token, uint8_t* done_out, BeamChunk* stat, uint2* cand, int sms,
                               cudaStream_t s) {
  // Long stretches save most of a stretch's fixed work, short ones keep the SMs even: one
  // round of the resident CTAs (four to an SM) while that is up to four steps each, else two.
  // 128256 logits, us by steps: 64 beams (4 are one round) 18.1 with one, 14.5 with two,
  // 13.3 with four, 15.0 with eight; 192 (11 and 6 steps) 28.0 with five, 27.6 with six, 28.9
  // with 11; 256 (16 and 8) 31.6 with five, 31.7 with eight, 32.7 with 16.
  const int rows = B * W, total = beam_chunks_most(V);
  auto steps = [&](int rounds) {
    const int c = std::max(1, std::min(total, rounds * 4 * sms / rows));
    return (total + c - 1) / c;
  };
  const int tiles = steps(1) <= 4 ? steps(1) : std::min(steps(2), 16);
  const int chunks = (total + tiles - 1) / tiles;
  ZSAA_LAUNCH(beam_scan_kernel, dim3(static_cast<unsigned>(rows) * static_cast<unsigned>(chunks)), dim3(kScanThreads), 0,
              s, logits, ld, V, K, chunks, tiles, done, stat, cand);
  auto merge_smem = [](int w, int k) {
    return w * k * 16 + (w > kSumWarps ? kMergeWarps : kSumWarps) * (2 * k + kMergeDepth * 64) * 8;
  };
  static OncePerDevice once;
  const cudaError_t e = set_smem_limit_once(once, beam_merge_kernel, merge_smem(kBeamMaxBeams, kBeamMaxKept));
  if (e != cudaSuccess) return e;
  ZSAA_LAUNCH(beam_merge_kernel, dim3(B), dim3(kMergeThreads), merge_smem(W, K), s, stat, cand, W, V, K, chunks, scores,
              done, eos, scores_out, parent, token, done_out);
  return cudaSuccess;
}

cudaError_t launch_beam_reorder(const PoolList& pools, int n_pages, int page_shift, int Hkv, int entry_bytes, int B,
                                int W, int K, const int32_t* parent, const int32_t* table, int32_t* table_out,
                                int cols, const int32_t* lens, int32_t* lens_out, const int32_t* fresh, int* status,
                                cudaStream_t s) {
  ReorderArgs a{};
  a.pools = pools;
  a.parent = parent, a.table = table, a.lens = lens, a.fresh = fresh;
  a.table_out = table_out, a.lens_out = lens_out;
  a.W = W, a.K = K, a.cols = cols, a.n_pages = n_pages, a.page_shift = page_shift, a.Hkv = Hkv;
  a.row_vecs = entry_bytes / 16;
  a.status = status;
  ZSAA_LAUNCH(beam_reorder_kernel, dim3(B * K, pools.n), dim3(256), 0, s, a);
  return cudaSuccess;
}

}  // namespace zsaa
