// Beam search over a batch: selection of the best continuations, and page tables
// that follow the selected beams.
//
// Selection.  Beam w of a batch element has a running score s_w and logits x_w over
// V tokens; continuation (w, v) has the total s_w + x_w[v] - lse(x_w), lse(x) =
// log sum exp(x).  The K largest totals are wanted; lse moves a whole beam, so a
// beam's own order is that of its logits and one pass over them is enough:
//   beam_scan_kernel   one chunk of one beam's logits per CTA, held in registers:
//                      its maximum, its sum of exponentials and its K best tokens;
//   beam_merge_kernel  one CTA per batch element: lse of every beam from the chunks'
//                      (m, s) pairs, totals in 64 bits, the K best of the chunks'.
// The logits are read once, which bounds large batches; few beams are bound by the
// two kernels' own chains.
//
// The K best without a sort: every warp publishes the eight best of its 32 lanes'
// maxima, and the K-th best published value T is a lower bound of the K-th best of
// all (at least K values reach it).  Only the few values that reach T are collected
// and ranked by counting.  Values are compared together with their place, lower
// place first, so that ties (a banned vocabulary is all -inf) collect no more than
// distinct values do; where more than the list holds reach T, the K-th best is
// found bit by bit instead.
#include "common.cuh"
#include "paged.cuh"

namespace zsaa {
namespace {

constexpr int kScanThreads = 256;
constexpr int kScanWarps = kScanThreads / 32;
constexpr int kMergeThreads = 512;
constexpr int kMergeWarps = kMergeThreads / 32;
constexpr int kPublish = 8;    // lane maxima that a warp publishes
constexpr int kListCap = 1024;  // collected values at most
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLog2eRest = static_cast<float>(1.4426950408889634 - static_cast<double>(kLog2e));

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

__device__ __forceinline__ double warp_sum_d(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Chunk c of row r: E values per thread.  A value's place is its token; a collected
// value is (key << 32 | ~token), so that a larger one is a better one.  NaN logits
// are ordered as -inf (their row's totals are all NaN).
template <int E>
__global__ void __launch_bounds__(kScanThreads)
    beam_scan_kernel(const float* __restrict__ logits, long long ld, int V, int K, int chunks,
                     const uint8_t* __restrict__ done, BeamChunk* __restrict__ stat, uint2* __restrict__ cand) {
  constexpr int CHUNK = kScanThreads * E;
  __shared__ uint64_t pub[kScanWarps * kPublish], list[kListCap];
  __shared__ uint64_t s_bound, s_best;
  __shared__ int s_count, s_bad, s_n[kScanWarps];
  __shared__ double s_sum[kScanWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = blockIdx.x / chunks, c = blockIdx.x % chunks;
  pdl_trigger();
  if (tid == 0) s_bound = 0, s_count = 0, s_bad = 0;
  pdl_wait();
  logits = after_wait(logits);
  done = after_wait(done);
  if (done != nullptr && done[row] != 0) return;  // its only continuation needs no logits
  const float* p = logits + static_cast<long long>(row) * ld;
  // 16-byte loads start `mis` values before the row, at the boundary below it
  const int mis = static_cast<int>((reinterpret_cast<uintptr_t>(p) >> 2) & 3);
  const int first = c * CHUNK - mis;  // token of the chunk's first place
  uint2* out = cand + (static_cast<size_t>(row) * chunks + c) * K;
  if (first >= V) {  // (only ever the row's last chunk)
    if (tid == 0) stat[static_cast<size_t>(row) * chunks + c] = BeamChunk{0.0, -INFINITY, 0};
    for (int i = tid; i < K; i += kScanThreads) out[i] = make_uint2(0, 0);
    return;
  }
  const bool edge = first < 0 || first + CHUNK > V;
  float v[E];
#pragma unroll
  for (int i = 0; i < E / 4; ++i) {
    const int t = first + (i * kScanThreads + tid) * 4;
    float4 f = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    if (t >= 0 && t <= V - 4) {
      f = __ldcs(reinterpret_cast<const float4*>(p + t));
    } else {
      if (t >= 0 && t < V) f.x = p[t];
      if (t + 1 >= 0 && t + 1 < V) f.y = p[t + 1];
      if (t + 2 >= 0 && t + 2 < V) f.z = p[t + 2];
      if (t + 3 >= 0 && t + 3 < V) f.w = p[t + 3];
    }
    v[4 * i] = f.x, v[4 * i + 1] = f.y, v[4 * i + 2] = f.z, v[4 * i + 3] = f.w;
  }
  auto token = [&](int i) { return first + ((i >> 2) * kScanThreads + tid) * 4 + (i & 3); };
  auto inside = [&](int i) { return !edge || (token(i) >= 0 && token(i) < V); };
  auto value = [&](int i) {
    return static_cast<uint64_t>(float_key(v[i])) << 32 | static_cast<uint32_t>(~token(i));
  };
  bool bad = false;
  float best = -INFINITY;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    bad |= !(v[i] < INFINITY);
    v[i] = fmaxf(v[i], -INFINITY);  // NaN -> -inf
    best = fmaxf(best, v[i]);
  }
  if (bad) s_bad = 1;  // (the same value from every thread that stores it)
  int at = -1;
#pragma unroll
  for (int i = E - 1; i >= 0; --i)
    if (v[i] == best && inside(i)) at = i;
  uint64_t mine = 0;
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (i == at) mine = value(i);
  for (int k = 0; k < kPublish; ++k) {
    const uint32_t hi = static_cast<uint32_t>(mine >> 32);
    const uint32_t top = __reduce_max_sync(0xffffffffu, hi);
    const uint32_t lo = __reduce_max_sync(0xffffffffu, hi == top ? static_cast<uint32_t>(mine) : 0u);
    const uint64_t w = static_cast<uint64_t>(top) << 32 | lo;
    if (lane == 0) pub[warp * kPublish + k] = top == 0 ? 0 : w;
    if (mine == w) mine = 0;
  }
  __syncthreads();
  if (tid < kScanWarps * kPublish) {
    const uint64_t x = pub[tid];
    int r = 0;
#pragma unroll 8
    for (int j = 0; j < kScanWarps * kPublish; ++j) r += pub[j] > x;
    if (x != 0 && r == 0) s_best = x;
    if (x != 0 && r == K - 1) s_bound = x;
  }
  __syncthreads();
  const float m = key_float(static_cast<uint32_t>(s_best >> 32));
  uint64_t bound = s_bound;
  const float bv = bound == 0 ? -INFINITY : key_float(static_cast<uint32_t>(bound >> 32));
  // sum of exp(x - m): a thread's values in 32 bits, the threads' sums in 64
  float s4[4] = {0.f, 0.f, 0.f, 0.f};
  // (x - m first: m log2(e) rounded to 32 bits would be off by more than the sum is;
  // log2(e) in two parts for the same reason)
  const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float d = v[i] - base;
    s4[i & 3] += ex2_fast(fmaf(d, kLog2e, d * kLog2eRest));
  }
  auto collect = [&](uint64_t from, float from_v) {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (v[i] >= from_v && inside(i) && value(i) >= from) {
        const int n = atomicAdd(&s_count, 1);
        if (n < kListCap) list[n] = value(i);
      }
  };
  collect(bound, bv);
  const double ws = warp_sum_d(static_cast<double>((s4[0] + s4[1]) + (s4[2] + s4[3])));
  if (lane == 0) s_sum[warp] = ws;
  __syncthreads();
  if (tid == 0) {
    double s = 0.0;
    for (int w = 0; w < kScanWarps; ++w) s += s_sum[w];
    stat[static_cast<size_t>(row) * chunks + c] = BeamChunk{m == -INFINITY ? 0.0 : s, m, s_bad};
  }
  int n = s_count;
  if (n > kListCap) {  // block-uniform: the K-th largest value, bit by bit
    bound = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t t = bound | (1ull << bit);
      int have = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) have += inside(i) && value(i) >= t;
      have = __reduce_add_sync(0xffffffffu, have);
      __syncthreads();  // the previous round's counts are read
      if (lane == 0) s_n[warp] = have;
      __syncthreads();
      int all = 0;
      for (int w = 0; w < kScanWarps; ++w) all += s_n[w];
      if (all >= K) bound = t;
    }
    __syncthreads();
    if (tid == 0) s_count = 0;
    __syncthreads();
    collect(bound, key_float(static_cast<uint32_t>(bound >> 32)));
    __syncthreads();
    n = s_count;
  }
  for (int i = tid; i < n; i += kScanThreads) {
    const uint64_t x = list[i];
    int r = 0;
    for (int j = 0; j < n; ++j) r += list[j] > x;
    if (r < K) out[r] = make_uint2(static_cast<uint32_t>(x >> 32), ~static_cast<uint32_t>(x));
  }
  for (int i = n + tid; i < K; i += kScanThreads) out[i] = make_uint2(0, 0);  // fewer tokens than K
}

// A continuation's rank: its total, then the lower beam, the higher logit, the lower token.
struct Rank {
  uint64_t total, rest;
  __device__ __forceinline__ bool operator>(const Rank& o) const {
    return total > o.total || (total == o.total && rest > o.rest);
  }
};
constexpr int kTokenBits = 26;
static_assert(kBeamMaxVocab == 1 << kTokenBits && kBeamMaxBeams == 64, "beam, logit and token share 64 bits");
__device__ __forceinline__ uint64_t rank_rest(int w, uint32_t key, int token) {
  return static_cast<uint64_t>(kBeamMaxBeams - 1 - w) << 58 | static_cast<uint64_t>(key) << kTokenBits |
         static_cast<uint64_t>(kBeamMaxVocab - 1 - token);
}

__device__ __forceinline__ uint64_t warp_max_u64(uint64_t v) {
  const uint32_t hi = static_cast<uint32_t>(v >> 32);
  const uint32_t top = __reduce_max_sync(0xffffffffu, hi);
  const uint32_t lo = __reduce_max_sync(0xffffffffu, hi == top ? static_cast<uint32_t>(v) : 0u);
  return static_cast<uint64_t>(top) << 32 | lo;
}
__device__ __forceinline__ Rank warp_max_rank(const Rank& r) {
  Rank w;
  w.total = warp_max_u64(r.total);
  w.rest = warp_max_u64(r.total == w.total ? r.rest : 0);
  return w;
}

__global__ void __launch_bounds__(kMergeThreads)
    beam_merge_kernel(const BeamChunk* __restrict__ stat, const uint2* __restrict__ cand, int W, int V, int K,
                      int chunks, const float* __restrict__ scores, const uint8_t* __restrict__ done, int eos,
                      float* __restrict__ scores_out, int32_t* __restrict__ parent, int32_t* __restrict__ token,
                      uint8_t* __restrict__ done_out) {
  __shared__ double s_lse[kBeamMaxBeams], s_score[kBeamMaxBeams];
  __shared__ uint8_t s_done[kBeamMaxBeams];
  __shared__ Rank pub[kMergeWarps * kPublish], list[kListCap], s_bound;
  __shared__ int s_count;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.x;
  pdl_trigger();
  if (tid == 0) s_bound = Rank{0, 0}, s_count = 0;
  pdl_wait();
  stat = after_wait(stat) + static_cast<size_t>(b) * W * chunks;
  cand = after_wait(cand) + static_cast<size_t>(b) * W * chunks * K;
  scores = after_wait(scores);
  done = after_wait(done);
  for (int w = warp; w < W; w += kMergeWarps) {
    const bool over = done != nullptr && done[b * W + w] != 0;
    double lse = 0.0;
    if (!over) {
      float m = -INFINITY;
      int bad = 0;
      for (int c = lane; c < chunks; c += 32) {
        m = fmaxf(m, stat[w * chunks + c].m);
        bad |= stat[w * chunks + c].bad;
      }
      m = warp_max(m);
      bad = __any_sync(0xffffffffu, bad);
      double s = 0.0;
      for (int c = lane; c < chunks; c += 32) {
        const BeamChunk st = stat[w * chunks + c];
        if (st.m != -INFINITY) s += st.s * exp(static_cast<double>(st.m) - static_cast<double>(m));
      }
      s = warp_sum_d(s);
      // no allowed token: every total is -inf (x - 0); a NaN or +inf logit: every total NaN
      lse = bad ? nan("") : m == -INFINITY ? 0.0 : static_cast<double>(m) + log(s);
    }
    if (lane == 0) {
      s_lse[w] = lse;
      s_score[w] = scores == nullptr ? 0.0 : static_cast<double>(scores[b * W + w]);
      s_done[w] = over;
    }
  }
  __syncthreads();
  const int n_all = W * chunks * K;
  // continuation i; total and rest 0 where there is none
  auto rank_of = [&](int i) {
    const int w = i / (chunks * K);
    uint32_t key;
    int tok;
    if (s_done[w]) {  // eos at no cost; the other tokens, in their order, are not allowed
      const int k = i - w * (chunks * K);
      if (k >= K || k >= V) return Rank{0, 0};
      tok = k == 0 ? eos : k - 1 < eos ? k - 1 : k;
      key = k == 0 ? 0x80000000u : 0x007fffffu;
    } else {
      const uint2 x = cand[i];
      if (x.x == 0) return Rank{0, 0};
      key = x.x;
      tok = static_cast<int>(x.y);
    }
    const double t = s_score[w] + (static_cast<double>(key_float(key)) - s_lse[w]);
    return Rank{double_key(t), rank_rest(w, key, tok)};
  };
  Rank mine{0, 0};
  for (int i = tid; i < n_all; i += kMergeThreads) {
    const Rank r = rank_of(i);
    if (r > mine) mine = r;
  }
  for (int k = 0; k < kPublish; ++k) {
    const Rank w = warp_max_rank(mine);
    if (lane == 0) pub[warp * kPublish + k] = w;
    if (mine.total == w.total && mine.rest == w.rest) mine = Rank{0, 0};
  }
  __syncthreads();
  if (tid < kMergeWarps * kPublish) {
    const Rank x = pub[tid];
    int r = 0;
    for (int j = 0; j < kMergeWarps * kPublish; ++j) r += pub[j] > x;
    if (x.rest != 0 && r == K - 1) s_bound = x;
  }
  __syncthreads();
  const Rank bound = s_bound;
  for (int i = tid; i < n_all; i += kMergeThreads) {
    const Rank r = rank_of(i);
    if (r.rest != 0 && !(bound > r)) {
      const int n = atomicAdd(&s_count, 1);
      if (n < kListCap) list[n] = r;
    }
  }
  __syncthreads();
  int n = s_count;
  if (n > kListCap) {  // block-uniform: one continuation after the other
    Rank last{~0ull, ~0ull};
    for (int k = 0; k < K; ++k) {
      Rank next{0, 0};
      for (int i = tid; i < n_all; i += kMergeThreads) {
        const Rank r = rank_of(i);
        if (last > r && r > next) next = r;
      }
      next = warp_max_rank(next);
      if (lane == 0) pub[warp] = next;
      __syncthreads();
      last = pub[0];
      for (int w = 1; w < kMergeWarps; ++w)
        if (pub[w] > last) last = pub[w];
      if (tid == 0) list[k] = last;
      __syncthreads();
    }
    n = K;
  }
  for (int i = tid; i < n; i += kMergeThreads) {
    const Rank x = list[i];
    int r = 0;
    for (int j = 0; j < n; ++j) r += list[j] > x;
    if (r >= K) continue;
    const int w = kBeamMaxBeams - 1 - static_cast<int>(x.rest >> 58);
    const int tok = kBeamMaxVocab - 1 - static_cast<int>(x.rest & (kBeamMaxVocab - 1));
    const size_t o = static_cast<size_t>(b) * K + r;
    scores_out[o] = key_double_to_float(x.total);
    parent[o] = w;
    token[o] = tok;
    if (done_out != nullptr) done_out[o] = s_done[w] || tok == eos;
  }
}

// One CTA per (slot, layer's K or V).  Slot j of batch element b continues beam p =
// parent[b][j]: it takes over the parent's whole pages; the partly filled page stays
// with the parent's first child, and a later child gets its entries copied into its
// own fresh page.
struct ReorderArgs {
  void* pool[2 * kReorderMaxLayers];  // K and V of each layer
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
  uint4* pool = static_cast<uint4*>(a.pool[blockIdx.y]);
  const uint4* s = pool + static_cast<size_t>(from) * a.Hkv * stride;
  uint4* d = pool + static_cast<size_t>(to) * a.Hkv * stride;
  for (int h = 0; h < a.Hkv; ++h)
    for (int i = tid; i < n; i += blockDim.x) d[static_cast<size_t>(h) * stride + i] = s[static_cast<size_t>(h) * stride + i];
}

int scan_values(int rows, int V, int sms) {
  // 32 values a thread where that gives every SM two chunks, else 8: one prompt's
  // beams would leave most SMs without work
  return static_cast<long long>(rows) * ((V + 3 + 32 * kScanThreads - 1) / (32 * kScanThreads)) >= 2LL * sms ? 32 : 8;
}

}  // namespace

int beam_chunks_most(int V) { return (V + 3 + 8 * kScanThreads - 1) / (8 * kScanThreads); }

int beam_chunks(int rows, int V, int sms) {
  const int chunk = scan_values(rows, V, sms) * kScanThreads;
  return (V + 3 + chunk - 1) / chunk;
}

cudaError_t launch_beam_select(const float* logits, long long ld, int B, int W, int V, const float* scores,
                               const uint8_t* done, int eos, int K, float* scores_out, int32_t* parent,
                               int32_t* token, uint8_t* done_out, BeamChunk* stat, uint2* cand, int sms,
                               cudaStream_t s) {
  const int rows = B * W, chunks = beam_chunks(rows, V, sms);
  const dim3 grid(static_cast<unsigned>(rows) * static_cast<unsigned>(chunks));
  if (scan_values(rows, V, sms) == 32)
    ZSAA_LAUNCH(beam_scan_kernel<32>, grid, dim3(kScanThreads), 0, s, logits, ld, V, K, chunks, done, stat, cand);
  else
    ZSAA_LAUNCH(beam_scan_kernel<8>, grid, dim3(kScanThreads), 0, s, logits, ld, V, K, chunks, done, stat, cand);
  ZSAA_LAUNCH(beam_merge_kernel, dim3(B), dim3(kMergeThreads), 0, s, stat, cand, W, V, K, chunks, scores, done, eos,
              scores_out, parent, token, done_out);
  return cudaSuccess;
}

cudaError_t launch_beam_reorder(const void* const* k, const void* const* v, int n_layers, int n_pages, int page_shift,
                                int Hkv, int entry_bytes, int B, int W, int K, const int32_t* parent,
                                const int32_t* table, int32_t* table_out, int cols, const int32_t* lens,
                                int32_t* lens_out, const int32_t* fresh, int* status, cudaStream_t s) {
  ReorderArgs a{};
  for (int l = 0; l < n_layers; ++l) {
    a.pool[2 * l] = const_cast<void*>(k[l]);
    a.pool[2 * l + 1] = const_cast<void*>(v[l]);
  }
  a.parent = parent, a.table = table, a.lens = lens, a.fresh = fresh;
  a.table_out = table_out, a.lens_out = lens_out;
  a.W = W, a.K = K, a.cols = cols, a.n_pages = n_pages, a.page_shift = page_shift, a.Hkv = Hkv;
  a.row_vecs = entry_bytes / 16;
  a.status = status;
  ZSAA_LAUNCH(beam_reorder_kernel, dim3(B * K, 2 * n_layers), dim3(256), 0, s, a);
  return cudaSuccess;
}

}  // namespace zsaa
