// Appending to a paged cache and attention over it.
//
// A cache is a pool of pages [n_pages, Hkv, page, hd] for keys and one for values; a
// sequence's table row lists its pages in order, entry i lies in page row[i / page].
// Appending rotates keys (and the call's queries) to their positions on the way, so
// keys are written once and the projection needs no position.
//
// Attention: sequence s of group g has n_q new entries, its last; query j sees the
// group's prefix and the sequence's entries i <= len - n_q + j.  Short tables take one launch
// (k_paged_mma.cu).  Else a prefix is read once for each tile of 16 or 128 of its group's query
// rows, in L2 as a rule after the first (paged.cuh has the decomposition), and the launch that
// joins adds the partial results.  The at most n_q - 1
// entries that only some of the queries see are added at the end of a query row, one by one
// and so without a mask: a value hidden from a query, finite or not, never enters its sums.
#include <algorithm>
#include <cmath>

#include "paged.cuh"

namespace zsaa {
namespace {

// ---------------------------------------------------------------- append

// RPC rows per CTA, kAppendThreads threads.  A thread handles 8 dims of a head's first
// half and the 8 that they pair with, so a rotation is thread-local; the row's sines
// and cosines (one set for all heads) go through shared memory.  A thread's first loads are
// out before the sines and the lookup of the entries.
// Angle: the position times the frequency in 2^-64 turns, modulo a turn, is one 64-bit
// product, exact for every 32-bit position.  The nearest quarter turn is taken off
// before the conversion to float, so sine and cosine are good to about 1e-7; to that the
// frequency's own rounding to 53 bits adds 2^-53 of the angle, 2^-22 at the farthest positions.
// Bound by bytes on prompts (8411 rows of 6144 bf16: 35 us, 5.8 TB/s; more units a thread in
// flight cost occupancy and up to twice that), by the chain table -> address -> store on
// single tokens (8 rows: 2.5 us).
constexpr int kAppendThreads = 256;

template <typename TI>
__device__ __forceinline__ void load8(const TI* p, float (&x)[8]) {
  if constexpr (sizeof(TI) == 2) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    x[0] = bf16lo(u.x), x[1] = bf16hi(u.x), x[2] = bf16lo(u.y), x[3] = bf16hi(u.y);
    x[4] = bf16lo(u.z), x[5] = bf16hi(u.z), x[6] = bf16lo(u.w), x[7] = bf16hi(u.w);
  } else {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
}
template <typename TO>
__device__ __forceinline__ void store8(TO* p, const float (&x)[8]) {
  if constexpr (sizeof(TO) == 2) {  // the one rounding
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                              pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  } else {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  }
}

__device__ __forceinline__ float2 turn_cos_sin(unsigned long long turn) {
  const unsigned quarter = static_cast<unsigned>((turn + (1ull << 61)) >> 62);
  const long long rest = static_cast<long long>(turn - (static_cast<unsigned long long>(quarter) << 62));
  float s, c;
  sincospif(static_cast<float>(rest) * 0x1p-63f, &s, &c);  // half turns, at most 1/4
  switch (quarter & 3) {
    case 0: return make_float2(c, s);
    case 1: return make_float2(-s, c);
    case 2: return make_float2(-c, -s);
    default: return make_float2(s, -c);
  }
}

template <typename TI, typename TO, int HD, int RPC>
__global__ void __launch_bounds__(kAppendThreads, RPC == 1 ? 1 : 8)
    append_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ RopeTurns turns) {
  constexpr int HALF = HD / 2, UNITS = HALF / 8;  // 8-dim pairs of a head
  constexpr int BATCH = RPC == 1 ? 2 : 1;  // units of a thread in flight
  __shared__ float2 cs[RPC][HALF];  // dim 8 u + j at j * UNITS + u: a warp's reads fall into different banks
  __shared__ long long s_at[RPC];  // element offset of the row's entry for head 0, or -1
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x;
  const int row0 = blockIdx.x * RPC, n = min(RPC, a.T - row0);
  const int h0 = a.q_out != nullptr ? 0 : a.Hq, per_row = (a.Hq + 2 * a.Hkv - h0) * UNITS, all = n * per_row;
  const TI* src = after_wait(static_cast<const TI*>(a.qkv));
  struct Unit {
    int r, h, c;  // row of the CTA, head, first dim
  };
  auto unit = [&](int i) {
    const int r = RPC == 1 ? 0 : static_cast<int>(static_cast<unsigned>(i) / static_cast<unsigned>(per_row)), k = i - r * per_row;
    return Unit{r, h0 + k / UNITS, (k % UNITS) * 8};
  };
  float x[BATCH][8], y[BATCH][8];
  auto load = [&](int base) {
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int i = base + b * kAppendThreads + tid;
      if (i >= all) continue;
      const Unit u = unit(i);
      const TI* p = src + static_cast<long long>(row0 + u.r) * a.ld + u.h * HD + u.c;
      load8(p, x[b]);
      load8(p + HALF, y[b]);
    }
  };
  load(0);
  const int32_t* pos = after_wait(a.pos);
  for (int i = tid; i < n * HALF; i += kAppendThreads) {
    const int r = i / HALF, c = i % HALF;
    cs[r][(c & 7) * UNITS + (c >> 3)] = turn_cos_sin(static_cast<unsigned long long>(static_cast<long long>(pos[row0 + r])) * turns.f[c]);
  }
  if (tid < n) {
    const int t = row0 + tid;
    int s = t, back = 1;  // back: 1 for the sequence's last row, 2 for the one before, ...
    if (a.cu_rows != nullptr) {
      const int32_t* cu = after_wait(a.cu_rows);
      int lo = -1, hi = a.S;  // the last sequence that starts at or before row t
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= t) lo = mid; else hi = mid;
      }
      s = lo;
      back = s >= 0 ? cu[s + 1] - t : 0;
    }
    long long at = -1;
    if (s >= 0 && back > 0) {  // not a row before the first sequence or behind the last
      const int e = max(after_wait(a.lens)[s], 0) - back;  // (of a negative length: below 0 as well)
      if (e >= 0) {
        if (e >> a.page_shift < a.cols) {
          const int page = after_wait(a.table)[static_cast<size_t>(s) * a.cols + (e >> a.page_shift)];
          if (page >= 0 && page < a.n_pages)
            at = (((static_cast<long long>(page) * a.Hkv) << a.page_shift) + (e & ((1 << a.page_shift) - 1))) * HD;
        }
        if (at < 0) atomicOr(a.status, kStatusBadIndex);
      }
    }
    s_at[tid] = at;
  }
  __syncthreads();
  for (int base = 0; base < all; base += BATCH * kAppendThreads) {
    if (base > 0) load(base);
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int i = base + b * kAppendThreads + tid;
      if (i >= all) continue;
      const Unit u = unit(i);
      const long long at = s_at[u.r];
      if (at < 0) continue;
      if (u.h < a.Hq + a.Hkv) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 w = cs[u.r][j * UNITS + (u.c >> 3)];
          const float p = x[b][j] * w.x - y[b][j] * w.y, q = y[b][j] * w.x + x[b][j] * w.y;
          x[b][j] = p;
          y[b][j] = q;
        }
      }
      TO* d;
      if (u.h < a.Hq) {
        d = static_cast<TO*>(a.q_out) + (static_cast<long long>(row0 + u.r) * a.Hq + u.h) * HD;
      } else {
        const bool key = u.h < a.Hq + a.Hkv;
        const int g = u.h - a.Hq - (key ? 0 : a.Hkv);
        d = static_cast<TO*>(key ? a.k : a.v) + at + ((static_cast<long long>(g) << a.page_shift) * HD);
      }
      store8(d + u.c, x[b]);
      store8(d + u.c + HALF, y[b]);
    }
  }
}

template <typename TI, typename TO, int HD>
cudaError_t run_append(const AppendArgs& a, const RopeTurns& t, int sms, cudaStream_t s) {
  // two rows per CTA share its prologue; fewer rows than would fill the SMs so go one by one
  if (a.T >= 8 * sms)
    ZSAA_LAUNCH(append_kernel<TI, TO, HD, 2>, dim3((a.T + 1) / 2), dim3(kAppendThreads), 0, s, a, t);
  else
    ZSAA_LAUNCH(append_kernel<TI, TO, HD, 1>, dim3(a.T), dim3(kAppendThreads), 0, s, a, t);
  return cudaSuccess;
}

// ---------------------------------------------------------------- joining the partial results

constexpr int kJoinThreads = 128;

// One warp per query row: the row's partials in the order of their keys, then the
// entries that the row sees and its sequence's earlier queries do not.  Bound by its chain
// of round trips to L2, some 900 clocks each, so there are three: everything about the
// row's sequence and, a lane per group, about its group; the log2 sums; the results, 8 at
// a time.
template <typename T, int HD>
__global__ void __launch_bounds__(kJoinThreads, 4)
    paged_join_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedWork wp,
                      const __grid_constant__ PagedWork ws) {
  const int lane = threadIdx.x & 31, Hq = a.Hkv * a.per;
  const int token = static_cast<int>(blockIdx.x), h = static_cast<int>(blockIdx.y) * (kJoinThreads / 32) + (threadIdx.x >> 5);
  pdl_trigger();
  if (h >= Hq) return;
  const int s = token / a.n_q, j = token - s * a.n_q, g = h / a.per;
  pdl_wait();
  const int len = paged_len(a.lens[s], a.cols << a.page_shift);
  const int own_per = ws.head[0], own_t = ws.head[1 + a.G + s - ws.e0];
  JoinParts shared{nullptr, nullptr, 0, 0};
  if (a.G > 0) {
    const int pre_per = wp.head[0];
    const PagedGroup x = paged_group_of(a, s, wp.head + 1 - wp.e0);
    if (x.g < 0) return;  // a row behind the last sequence stays as it was
    shared = join_prefix(a, wp, x, pre_per, s, g, j * a.per + h % a.per, HD);
  }
  const PagedEntry mine{max(0, len - (a.n_q - 1)), a.n_q * a.per, s};
  const JoinParts own = join_parts(a, ws, a.G + s, mine, own_per, own_t, g, j * a.per + h % a.per, HD);

  PagedRows<HD, 1> x{};
  x.rr[0] = j * a.per + h % a.per;
  x.m[0] = -INFINITY;
  paged_add_parts<T, HD, 1, 8>(x, {shared}, {own});
  paged_finish<T, HD, 1>(a, s, g, x);
}

// ---------------------------------------------------------------- launches

long long items_of(const PagedArgs& a, int mt, bool prefixes, bool sequences) {
  const long long row = static_cast<long long>(a.n_q) * a.per;
  long long n = 0;
  if (prefixes) n += (a.S * row / mt + a.G) * a.Hkv;
  if (sequences) n += static_cast<long long>(a.S) * ((row + mt - 1) / mt) * a.Hkv;
  return n;
}
long long units_of(const PagedArgs& a, int mt, int bn, int lead) {
  const long long row = static_cast<long long>(a.n_q) * a.per;
  const long long pk = (static_cast<long long>(a.pcols) << a.page_shift) / bn + 1 + lead;
  const long long sk = (static_cast<long long>(a.cols) << a.page_shift) / bn + 1 + lead;
  return (a.S * row / mt + a.G) * a.Hkv * pk + a.S * ((row + mt - 1) / mt) * a.Hkv * sk;
}

// Fills in a launch's share of the workspace from *at on and moves it.
PagedWork work_share(const PagedArgs& a, const PagedTiles& t, bool prefixes, bool sequences, int hd, uintptr_t* at) {
  auto take = [&](size_t bytes) {
    const uintptr_t p = *at;
    *at += (bytes + 255) & ~static_cast<size_t>(255);
    return p;
  };
  PagedWork w{};
  w.e0 = prefixes ? 0 : a.G;
  w.e1 = sequences ? a.G + a.S : a.G;
  w.min_units = t.min_units;
  w.lead = t.lead;
  while ((1 << w.mt_shift) < t.mt) ++w.mt_shift;
  while ((1 << w.bn_shift) < t.bn) ++w.bn_shift;
  const size_t slots = static_cast<size_t>(t.ctas) + static_cast<size_t>(items_of(a, t.mt, prefixes, sequences));
  w.head = reinterpret_cast<int*>(take(sizeof(int) * (1 + static_cast<size_t>(w.e1 - w.e0))));
  w.lse2 = reinterpret_cast<float*>(take(sizeof(float) * slots * t.mt));
  w.o = reinterpret_cast<float*>(take(sizeof(float) * slots * t.mt * hd));
  return w;
}

constexpr int kMostSms = 256;  // the workspace holds a device of up to this many SMs

// The attention launches of a call: which kernel takes the prefixes, which the sequences
// (one launch where it is the same), and their shares of the workspace.
struct Launches {
  int n;
  bool own;  // the sequences' own entries belong to the launch that joins
  bool tc[2];
  PagedTiles tiles[2];
  PagedWork work[2];
  size_t bytes;
  long long most;  // items and units that number the slots and the line
};

// The 128-row tiles take entries whose 16-row tiles would have more than `blocks` blocks of
// 64 keys to a CTA (304 CTAs with heads of 128 dims, 456 with 64: two and three to each of the
// 152 SMs the rules were measured on; by the tables' sizes).
// Up to 16 rows there is one 16-row tile and nothing to gain.  Six blocks where that saves
// or costs no launch (us, 16-row and 128-row tiles, 8 heads of 128 dims): 24 sequences of 4
// queries in 3 groups with 300 own entries, 512 keys 24 and 26, 1024 31 and 29, 2048 37 and 32,
// 8192 104 and 56; 62 of 5 in one group, 512 58 and 43, 2048 93 and 50; 128 of one in 4 groups
// and 300 own, which the joining launch then has, 512 46 and 54, 2048 58 and 60, 8192 131 and
// 84; with 64 dims the first 21 and 21 at 1024, 24 and 22, 60 and 40.  Forty where the
// sequences' own entries, too many for the joining launch, then need a launch of their own:
// the first with 1500 own 2048 keys 48 and 59, 4096 63 and 64, 8192 106 and 81; with 64 dims
// 31 and 37, 40 and 43, 66 and 55.  None where the sequences take 128-row tiles: 10 of 5 with
// 1200 own, 64 dims, 2048 keys 28 and 18.
bool many_rows(int hd, long long row_tiles, long long rows, long long keys, int heads, int blocks) {
  return rows > 16 && row_tiles * heads * (keys / 64) > blocks * (hd == 128 ? 304 : 456);
}

// Calls that one CTA for each sequence, KV head and tile of 16 rows does at once, without
// a plan and partial results.  Measured by the tables' sizes against the split over all SMs
// (us, 8 KV heads of 128 dims, bf16, 4 rows to a head): 4 sequences of 512 keys 6.3 and 9.2, of
// 1024 9.5 and 9.6, of 2048 16 and 12; 16 of 1024 14 and 19; 64 of 1024 47 and 52, of 2048 86
// and 90; 256 of 2048 311 and 338.  20 rows: 8 of 1024 12 and 16, 62 of 1024 73 and 68.  32 rows:
// 16 of 1024 23 and 28, 128 of 1024 147 and 147, of 2048 263 and 227.  64 rows, 16 of 256: 41 and
// 35, with 64 dims 28 and 33; of 1024 46 and 38.  A shared prefix is read again for every
// sequence: 16 in 4 groups, 1024 keys 11 and 13, 2048 18 and 16; 64 in 8, 256 14 and 19, 512 21
// and 18, 1024 34 and 24; 62 of 20 rows in 8, 512 45 and 45, 1024 73 and 53.
// In float32: 4 sequences of 256 keys 9.5 and 12, 512 16 and 12, with 32 dims 4.9 and 8.0 and at
// 1024 12 and 9.8; 16 of 1024 31 and 40; 64 of 1024 105 and 118, with 32 dims 49 and 40; 62 of 20
// rows 213 and 232.  With groups: 16 in 4, 256 11 and 16, 512 17 and 18; 64 in 8, 128 18 and 26,
// 256 30 and 26, with 32 dims 16 and 14, 27 and 17 at 512; 62 of 20 rows in 8, 256 68 and 86.
// The rules are coarser than these figures and give some of them away: 4% at 64 sequences of
// 2048 (split), 7% at 62 of 20 rows and 1024 keys (direct), and most, a fifth, at 64 float32
// sequences of 1024 with 32 dims (direct).
long long direct_ctas(const PagedArgs& a) {
  return static_cast<long long>(a.S) * a.Hkv * ((static_cast<long long>(a.n_q) * a.per + 15) / 16);
}
// The sequences' own entries in bf16, alone or in the launch that joins them with the
// prefixes' partial results.  That launch against two, after 128-row tiles, 300 entries: 24
// sequences of 4 queries 36 and 44 us with 2048 keys to a prefix, with 64 dims 23 and 30; 64
// sequences of 600 and a prefix of 32000 95 and 103; 8 of 8 queries, 64 rows, 1024 27 and 35.
// (128 sequences of one query with 64 dims: 48 and 44.)  After 16-row tiles, which take
// both kinds of entries in one launch, it gains nothing: 32 sequences in 8 groups 22 and 20.
bool own_in_one(const PagedArgs& a, int hd) {
  const long long keys = static_cast<long long>(a.cols) << a.page_shift, rows = static_cast<long long>(a.n_q) * a.per;
  if (a.Hkv * ((rows + 15) / 16) > 65535) return false;  // the grid's second dimension
  if (rows > 32) return (hd == 64 || a.G > 0) && keys <= 512;
  return keys <= 1024 || (rows <= 16 && direct_ctas(a) >= 4 * 304);
}
bool direct_call(const PagedArgs& a, bool bf16, int hd) {
  const long long keys = static_cast<long long>(a.cols + a.pcols) << a.page_shift;
  if (a.Hkv * ((static_cast<long long>(a.n_q) * a.per + 15) / 16) > 65535) return false;
  if (!bf16 && a.G == 0) return keys * hd <= 16384 || (direct_ctas(a) >= 96 && keys <= 1024);
  if (!bf16) return keys <= 256 || keys * hd <= 16384;
  return a.G == 0 ? own_in_one(a, hd) : keys <= (direct_ctas(a) <= 152 ? 1024 : 512);
}

Launches launches_of(const PagedArgs& a, int dtype, int hd, int sms, void* ws) {
  Launches r{};
  const long long row = static_cast<long long>(a.n_q) * a.per;
  const bool bf = dtype == ZSAA_BF16;
  const bool own = bf && a.G > 0 && own_in_one(a, hd);
  const bool tc_seq = bf && many_rows(hd, a.S * ((row + 15) / 16), row, static_cast<long long>(a.cols) << a.page_shift, a.Hkv, 6);
  const bool tc_pre = tc_seq || (bf && a.G > 0 &&
                                 many_rows(hd, std::max(a.S * row / 16, static_cast<long long>(a.G)), a.S * row / a.G,
                                           static_cast<long long>(a.pcols) << a.page_shift, a.Hkv, own ? 6 : 40));
  r.own = own && tc_pre;
  r.n = tc_seq == tc_pre || r.own ? 1 : 2;
  uintptr_t at = reinterpret_cast<uintptr_t>(ws);
  for (int i = 0; i < r.n; ++i) {
    const bool pre = i == 0, seq = i == r.n - 1 && !r.own;
    r.tc[i] = pre ? tc_pre : tc_seq;
    r.tiles[i] = r.tc[i] ? paged_tc_tiles(sms) : paged_mma_tiles(dtype, hd, sms);
    r.work[i] = work_share(a, r.tiles[i], pre, seq, hd, &at);
    const long long slots = items_of(a, r.tiles[i].mt, pre, seq) + r.tiles[i].ctas;
    const long long units = units_of(a, r.tiles[i].mt, r.tiles[i].bn, r.tiles[i].lead);
    r.most = std::max(r.most, std::max(slots, units));
  }
  r.bytes = at - reinterpret_cast<uintptr_t>(ws);
  return r;
}

template <typename T, int HD>
cudaError_t run_paged_attention(const PagedArgs& a, void* ws, int sms, cudaStream_t s) {
  constexpr int dtype = sizeof(T) == 4 ? ZSAA_F32 : ZSAA_BF16;
  if (direct_call(a, dtype == ZSAA_BF16, HD)) return launch_paged_direct(a, nullptr, dtype, HD, s);
  const Launches r = launches_of(a, dtype, HD, std::min(sms, kMostSms), ws);
  for (int i = 0; i < r.n; ++i) {
    const cudaError_t e = r.tc[i] ? launch_paged_tc(a, r.work[i], HD, r.tiles[i].ctas, s)
                                  : launch_paged_mma(a, r.work[i], dtype, HD, r.tiles[i].ctas, s);
    if (e != cudaSuccess) return e;
  }
  if (r.own) return launch_paged_direct(a, &r.work[0], dtype, HD, s);
  const int heads = a.Hkv * a.per, per_cta = kJoinThreads / 32;
  ZSAA_LAUNCH(paged_join_kernel<T, HD>, dim3(a.S * a.n_q, (heads + per_cta - 1) / per_cta), dim3(kJoinThreads), 0, s, a, r.work[0], r.work[r.n - 1]);
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_paged_append(const AppendArgs& a, int in_dtype, int dtype, int hd, float theta, int sms,
                                cudaStream_t s) {
  // the last call's frequencies: a model's calls all have the same
  thread_local RopeTurns t{};
  thread_local float t_theta = 0.f;
  thread_local int t_hd = 0;
  if (theta != t_theta || hd != t_hd) {
    for (int c = 0; c < hd / 2; ++c) {
      const double f = std::pow(static_cast<double>(theta), -2.0 * c / hd) / 6.283185307179586476925;
      t.f[c] = static_cast<unsigned long long>(std::ldexp(f, 64));
    }
    t_theta = theta;
    t_hd = hd;
  }
  if (dtype == ZSAA_F32) {
    if (hd == 32) return run_append<float, float, 32>(a, t, sms, s);
    if (hd == 64) return run_append<float, float, 64>(a, t, sms, s);
    if (hd == 128) return run_append<float, float, 128>(a, t, sms, s);
  } else if (in_dtype == ZSAA_F32) {
    if (hd == 64) return run_append<float, bf16, 64>(a, t, sms, s);
    if (hd == 128) return run_append<float, bf16, 128>(a, t, sms, s);
  } else {
    if (hd == 64) return run_append<bf16, bf16, 64>(a, t, sms, s);
    if (hd == 128) return run_append<bf16, bf16, 128>(a, t, sms, s);
  }
  return cudaErrorInvalidValue;
}

size_t paged_attention_workspace(const PagedArgs& a, int dtype, int hd) {
  const Launches r = launches_of(a, dtype, hd, kMostSms, nullptr);
  return r.most >= 0x3fffffff ? 0 : r.bytes;
}

cudaError_t launch_paged_attention(const PagedArgs& a, int dtype, int hd, void* ws, int sms, cudaStream_t s) {
  if (dtype == ZSAA_F32) {
    if (hd == 32) return run_paged_attention<float, 32>(a, ws, sms, s);
    if (hd == 64) return run_paged_attention<float, 64>(a, ws, sms, s);
    if (hd == 128) return run_paged_attention<float, 128>(a, ws, sms, s);
  } else {
    if (hd == 64) return run_paged_attention<bf16, 64>(a, ws, sms, s);
    if (hd == 128) return run_paged_attention<bf16, 128>(a, ws, sms, s);
  }
  return cudaErrorInvalidValue;
}

}  // namespace zsaa
