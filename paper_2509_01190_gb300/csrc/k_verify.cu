// Verification of drafted tokens against the target's probabilities, and the token that follows.
//
// Sequence s has n drafts x_j, n + 1 rows of target logits and n of draft logits, a temperature
// T and numbers u_0 .. u_n in [0, 1).  With p_j and q_j the softmax of the rows over T, draft j
// stands where u_j q_j(x_j) < p_j(x_j) and all before it stand.  The token behind the last one
// that stands is drawn from r = max(p - q, 0) at a refused draft, from p behind the last draft:
// the first token t with r_0 + .. + r_t > u_n (r_0 + .. + r_V-1).  The tokens are then
// distributed as the target's own.
//
//   verify_scan_kernel    one stretch of one row per CTA: its maximum and the sum of its
//                         exponentials.  Bound by the logits' bytes.
//   verify_finish_kernel  which drafts stand; then the rows at which a sequence stops again, a
//                         slice per CTA, and its last CTA finds the token.
//
// What decides a draft is one comparison of two quotients, off by about 1e-8 with sums of
// float32 exponentials.  What decides a token is where u_n falls among V borders, some 1e-5
// apart and closer: a running sum that is off by 1e-9 picks the wrong token every few thousand
// calls.  So the rows at which a sequence stops are gone through again with exponentials as
// pairs of floats, good to about 2^-37, and sums in pairs and in 64 bits.
//
// One pass does it, although the residual needs the sums of both rows: with E the exponentials,
// Z their exact sums and c0 the quotient Z_p / Z_q as the scan has it, the pass adds up
//   D_i = E_p,i - c0 E_q,i        over all tokens, and
//   A = sum D_i, B = sum E_q,i    over a group's tokens with D_i > 0.
// The exact quotient is c0 + k with k = sum D / Z_q, some 2^-24 of it, so a group's residual is
// A - k B; tokens whose D_i changes its sign with k are off by 2^-24 of a 2^-24th of them.
#include <algorithm>
#include <cmath>

#include "common.cuh"
#include "paged.h"

namespace zsaa {
namespace {

constexpr float kMinTemperature = 0x1p-64f, kMaxTemperature = 0x1p64f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

struct Temperature {
  float t;
  bool greedy, bad;
};
__device__ __forceinline__ Temperature temperature_of(const VerifyArgs& a, int s) {
  if (a.temperature == nullptr) return Temperature{1.f, false, false};
  const float t = after_wait(a.temperature)[s];
  return Temperature{t, t >= 0.f && t < kMinTemperature, !(t >= 0.f && t <= kMaxTemperature)};
}

__device__ __forceinline__ float log2e_over(float t) { return 1.44269504088896340736f / t; }

// drafts of sequence s before the first that is no token
// (whole warps)
__device__ __forceinline__ int drafts_of(const VerifyArgs& a, int s) {
  const int lane = threadIdx.x & 31;
  const int x = lane < a.n ? after_wait(a.drafts)[static_cast<size_t>(s) * a.n + lane] : -1;
  return __ffs(__ballot_sync(0xffffffffu, x < 0 || x >= a.V)) - 1;  // (lane 31 has no draft)
}

// ---------------------------------------------------------------- the rows' maxima and sums

constexpr int kScanThreads = 256, kScanValues = 32, kScanTokens = kScanThreads * kScanValues;

template <typename T>
__device__ __forceinline__ void load16(const T* p, float* x) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  if constexpr (sizeof(T) == 2) {
    x[0] = bf16lo(u.x), x[1] = bf16hi(u.x), x[2] = bf16lo(u.y), x[3] = bf16hi(u.y);
    x[4] = bf16lo(u.z), x[5] = bf16hi(u.z), x[6] = bf16lo(u.w), x[7] = bf16hi(u.w);
  } else {
    x[0] = __uint_as_float(u.x), x[1] = __uint_as_float(u.y), x[2] = __uint_as_float(u.z), x[3] = __uint_as_float(u.w);
  }
}

// Row r of sequence s: target row r for r <= n, else draft row r - n - 1.
template <typename T>
__device__ __forceinline__ const T* row_of(const VerifyArgs& a, int s, int r) {
  if (r <= a.n) return after_wait(static_cast<const T*>(a.target)) + (static_cast<long long>(s) * (a.n + 1) + r) * a.ld;
  return after_wait(static_cast<const T*>(a.draft)) + (static_cast<long long>(s) * a.n + (r - a.n - 1)) * a.draft_ld;
}

// (64-bit floats are left out of both kernels: the SM does two of their operations a clock.)
constexpr float kSumScale = 0x1p36f;  // a stretch's sum, at most 2^13, in units of 2^-36

// Sum over the warp of values in [0, 2^50) (two 32-bit reductions of 25 bits each).
__device__ __forceinline__ unsigned long long warp_sum_u50(unsigned long long v) {
  const unsigned lo = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(v) & 0x1ffffffu);
  const unsigned hi = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(v >> 25));
  return (static_cast<unsigned long long>(hi) << 25) + lo;
}

// Every warp takes its sum against its own maximum, so the warps meet once, at the end.
template <typename T>
__global__ void __launch_bounds__(kScanThreads, 4) verify_scan_kernel(const __grid_constant__ VerifyArgs a, int rows) {
  constexpr int VEC = 16 / sizeof(T), VECS = kScanValues / VEC;
  __shared__ float s_top[kScanThreads / 32];
  __shared__ unsigned long long s_sum[kScanThreads / 32];
  __shared__ int s_first[kScanThreads / 32];
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const unsigned item = blockIdx.x / static_cast<unsigned>(a.chunks);
  const int chunk = static_cast<int>(blockIdx.x - item * a.chunks);
  const int s = static_cast<int>(item / static_cast<unsigned>(rows)), r = static_cast<int>(item - s * static_cast<unsigned>(rows));
  if (r == 0 && chunk == 0 && tid == 0) a.done[s] = 0;
  const Temperature t = temperature_of(a, s);
  const bool is_draft = r > a.n;
  if (t.bad || (t.greedy && is_draft)) return;  // rows that decide nothing
  const int j = is_draft ? r - a.n - 1 : r;
  if (j > 0 || is_draft) {
    const int have = drafts_of(a, s);
    if (j > have || (is_draft && j == have)) return;
  }
  const T* row = row_of<T>(a, s, r);
  // the stretch starts on a 16-byte boundary, before the row's first token for the first one
  const int lead = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
  const int t0 = chunk * kScanTokens - lead;
  float x[kScanValues];
#pragma unroll
  for (int k = 0; k < VECS; ++k) {
    const int at = t0 + (k * kScanThreads + tid) * VEC;
    if (at >= 0 && at <= a.V - VEC) {
      load16(row + at, x + k * VEC);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[k * VEC + i] = at + i >= 0 && at + i < a.V ? to_f<T>(row[at + i]) : -INFINITY;
    }
  }
  float top = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int k = 0; k < kScanValues; ++k) {
    top = fmaxf(top, x[k]);
    bad |= !(x[k] < INFINITY);
  }
  top = warp_max(top);
  const float c = log2e_over(t.t);
  unsigned long long total = 0;
  int first = a.V;
  if (t.greedy) {
#pragma unroll
    for (int k = kScanValues - 1; k >= 0; --k) {
      const int at = t0 + ((k / VEC) * kScanThreads + tid) * VEC + k % VEC;
      if (x[k] == top && at >= 0 && at < a.V) first = at;
    }
    first = __reduce_min_sync(0xffffffffu, first);
  } else {
    const float ref = top == -INFINITY ? 0.f : top;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kScanValues; ++k) sum[k & 3] += ex2((x[k] - ref) * c);
    // (bad rows have any sum)
    total = warp_sum_u50(static_cast<unsigned long long>(fminf((sum[0] + sum[1]) + (sum[2] + sum[3]), 64.f) * kSumScale));
  }
  if (lane == 0) s_top[warp] = top, s_sum[warp] = total, s_first[warp] = first;
  bad = __syncthreads_or(bad) != 0;
  if (warp == 0) {
    const bool in = lane < kScanThreads / 32;
    top = in ? s_top[lane] : -INFINITY;
    const float all = warp_max(top);
    total = in && top > -INFINITY ? static_cast<unsigned long long>(static_cast<float>(s_sum[lane]) * ex2((top - all) * c)) : 0;
    VerifyChunk out;
    out.sum = static_cast<long long>(warp_sum_u50(total));
    out.top = all;
    out.first = __reduce_min_sync(0xffffffffu, in && top == all ? s_first[lane] : a.V);
    if (bad) out.first = -1;
    if (lane == 0) a.stat[(static_cast<size_t>(s) * rows + r) * a.chunks + chunk] = out;
  }
}

// ---------------------------------------------------------------- exponentials as pairs of floats

struct Pair {
  float h, l;
};

// exp((x - m) / T) = 2^y: y = (x - m) log2(e) / T with its rounding errors kept, cut into
// k / 32 and a rest f of at most 1/64; 2^(k/32) from a table of pairs, 2^f by its series, whose
// first term is a pair too (|f ln 2| <= 0.0109: the terms from the second on are below 2^-14 and
// their float32 errors below 2^-37, as is the first one left out).  0 below 2^-125.
struct MassRow {
  float m, ch, cl;  // the row's maximum; log2(e) / T
};
__device__ __forceinline__ MassRow mass_row(float m, float t) {
  constexpr float kLog2eH = 1.44269502162933349609375f;
  constexpr float kLog2eL = static_cast<float>(1.4426950408889634074 - static_cast<double>(kLog2eH));
  const float ch = kLog2eH / t;
  return MassRow{m, ch, (fmaf(-ch, t, kLog2eH) + kLog2eL) / t};
}
__device__ __forceinline__ Pair mass(float x, const MassRow& r, const float* table_h, const float* table_l) {
  constexpr float kLn2H = 0.693147182464599609375f;  // ln 2 rounded to float, and what that leaves
  constexpr float kLn2L = static_cast<float>(0.69314718055994530942 - static_cast<double>(kLn2H));
  const float d = x - r.m, b = d - x;
  const float de = (x - (d - b)) + (-r.m - b);  // what rounding took off x - m
  const float y = __fmul_rn(d, r.ch);  // (products whose rounding is kept are not fused into what follows)
  const float ye = fmaf(d, r.ch, -y) + fmaf(d, r.cl, de * r.ch);
  const float magic = fmaf(y, 32.f, 0x1.8p23f);
  const int k = __float_as_int(magic) - __float_as_int(0x1.8p23f);
  const float f = fmaf(magic - 0x1.8p23f, -0.03125f, y);
  const float g = __fmul_rn(f, kLn2H);
  const float ge = fmaf(f, kLn2H, -g) + fmaf(f, kLn2L, ye * kLn2H);
  const float w = g + ge;
  const float rest = ge + w * w * fmaf(w, fmaf(w, 1.f / 24.f, 1.f / 6.f), 0.5f);
  const float th = table_h[k & 31], tl = table_l[k & 31];
  const float ph = __fmul_rn(th, g);
  const float pl = fmaf(th, g, -ph) + fmaf(th, rest, fmaf(tl, g, tl));
  const float h = th + ph, l = (ph - (h - th)) + pl;
  const float scale = __int_as_float((max(k >> 5, -126) + 127) << 23);
  return y > -125.f ? Pair{h * scale, l * scale} : Pair{0.f, 0.f};
}

// arithmetic of pairs (products whose rounding is kept are not fused into what follows)
__device__ __forceinline__ void add(Pair& s, float h, float l) {
  const float t = s.h + h, b = t - s.h;
  s.l += ((s.h - (t - b)) + (h - b)) + l;
  s.h = t;
}
__device__ __forceinline__ Pair mul(const Pair& a, const Pair& b) {
  const float h = __fmul_rn(a.h, b.h);
  return Pair{h, fmaf(a.h, b.h, -h) + fmaf(a.h, b.l, a.l * b.h)};
}
__device__ __forceinline__ Pair sub(const Pair& a, const Pair& b) {
  const float h = a.h - b.h, c = h - a.h;
  return Pair{h, ((a.h - (h - c)) + (-b.h - c)) + (a.l - b.l)};
}
__device__ __forceinline__ Pair div(const Pair& a, const Pair& b) {
  const float h = a.h / b.h;
  return Pair{h, (fmaf(-h, b.h, a.h) + fmaf(-h, b.l, a.l)) / b.h};
}
__device__ __forceinline__ Pair warp_sum_pair(Pair v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float h = __shfl_xor_sync(0xffffffffu, v.h, o), l = __shfl_xor_sync(0xffffffffu, v.l, o);
    add(v, h, l);
  }
  return v;
}
__device__ __forceinline__ Pair pair_of(long long v, float unit) {
  const float h = __ll2float_rn(v);
  return Pair{h * unit, __ll2float_rn(v - __float2ll_rn(h)) * unit};
}
// in units of 1 / scale
__device__ __forceinline__ long long fixed(const Pair& v, float scale) {
  return __float2ll_rn(v.h * scale) + __float2ll_rn(v.l * scale);
}
__device__ __forceinline__ long long warp_sum_ll(long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// ---------------------------------------------------------------- decisions and the token

constexpr int kFinishThreads = 256, kFinishWarps = kFinishThreads / 32;
constexpr int kGroupLeast = 128, kGroupMost = 1024;  // tokens of a warp, whose sums are kept

enum { kFromTarget = 0, kWithout = 1, kResidual = 2 };  // r = p; p without token x; max(p - q, 0)

struct RowStat {
  Pair sum;
  float top;
  int first;
  int ok;  // the row has a distribution
};

// u q(x) < p(x) from the logits alone, where the exponentials are too small for float pairs
__device__ __noinline__ bool stands_far(float u, float xp, float xq, float t, const RowStat& p, const RowStat& q) {
  auto log_of = [t](float x, const RowStat& r) {
    return (static_cast<double>(x) - static_cast<double>(r.top)) / t - log(static_cast<double>(r.sum.h) + static_cast<double>(r.sum.l));
  };
  const double lp = log_of(xp, p), lq = log_of(xq, q);
  return lp > -INFINITY && (lq == -INFINITY || u < exp(lp - lq));
}

__device__ __forceinline__ VerifyGroup load_group(const VerifyGroup* p) {
  const longlong2 x = __ldcg(reinterpret_cast<const longlong2*>(p));
  VerifyGroup g;
  g.a = x.x;
  g.d = x.y;
  g.b = __ldcg(&p->b);
  return g;
}

// floor(u total), u in [0, 1)
__device__ __forceinline__ long long goal_of(float u, long long total) {
  int e;
  const float m = frexpf(u, &e);  // u = m 2^e, m 2^24 a whole number
  const unsigned __int128 v = static_cast<unsigned __int128>(static_cast<unsigned>(m * 0x1p24f)) * static_cast<unsigned long long>(total);
  return 24 - e > 127 ? 0 : static_cast<long long>(v >> (24 - e));
}

template <typename T>
__global__ void __launch_bounds__(kFinishThreads, 4)
    verify_finish_kernel(const __grid_constant__ VerifyArgs a, int rows, int ctas, int group, float unit) {
  __shared__ float table_h[32], table_l[32];
  __shared__ RowStat stat[2 * kVerifyMaxDrafts + 1];
  __shared__ int s_stands[kVerifyMaxDrafts + 1];
  __shared__ long long s_part[kFinishWarps], s_before;
  __shared__ int s_first[kFinishWarps], s_some[kFinishWarps], s_group, s_last;
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int s = static_cast<int>(blockIdx.x) / ctas, cta = static_cast<int>(blockIdx.x) - s * ctas;
  if (tid < 32) {
    const double e = exp2(tid / 32.0);
    table_h[tid] = static_cast<float>(e);
    table_l[tid] = static_cast<float>(e - static_cast<double>(table_h[tid]));
  }
  __syncthreads();
  pdl_wait();
  const Temperature t = temperature_of(a, s);
  const int n = drafts_of(a, s);
  const bool lookup = a.draft == nullptr, soft = !t.greedy && !t.bad;
  const int4* chunks = after_wait(reinterpret_cast<const int4*>(a.stat)) + static_cast<size_t>(s) * rows * a.chunks;
  auto chunk_at = [&](int r, int i) {
    const int4 v = chunks[static_cast<size_t>(r) * a.chunks + i];
    VerifyChunk c;
    c.sum = static_cast<long long>(static_cast<unsigned long long>(static_cast<unsigned>(v.y)) << 32 | static_cast<unsigned>(v.x));
    c.top = __int_as_float(v.z);
    c.first = v.w;
    return c;
  };

  // every row that may decide something: its maximum and its sum
  for (int r = warp; r < rows; r += kFinishWarps) {
    const bool is_draft = r > a.n;
    RowStat out{{0.f, 0.f}, -INFINITY, a.V, 0};
    if (!t.bad && (is_draft ? !t.greedy && r - a.n - 1 < n : r <= n)) {
      bool bad = false;
      for (int i = lane; i < a.chunks; i += 32) {
        const VerifyChunk c = chunk_at(r, i);
        out.top = fmaxf(out.top, c.top);
        bad |= c.first < 0;
      }
      out.top = warp_max(out.top);
      if (soft) {
        const MassRow m = mass_row(out.top, t.t);
        for (int i = lane; i < a.chunks; i += 32) {
          const VerifyChunk c = chunk_at(r, i);
          const Pair v = mul(pair_of(c.sum, 1.f / kSumScale), mass(c.top, m, table_h, table_l));
          if (c.top > -INFINITY) add(out.sum, v.h, v.l);
        }
        out.sum = warp_sum_pair(out.sum);
      } else {
        for (int i = lane; i < a.chunks; i += 32) {
          const VerifyChunk c = chunk_at(r, i);
          if (c.top == out.top) out.first = min(out.first, c.first);
        }
        out.first = __reduce_min_sync(0xffffffffu, out.first);
      }
      out.ok = !__any_sync(0xffffffffu, bad) && out.top > -INFINITY;
    }
    if (lane == 0) stat[r] = out;
  }
  __syncthreads();
  auto logit = [&](int r, int x) { return to_f<T>(row_of<T>(a, s, r)[x]); };
  // log p of a token of row r with the logit x: (x - top) / t - log(sum), the rounding errors of
  // each kept: log(sum) = g + log(sum exp(-g)) with g near it, and the latter is its argument less 1
  auto log_p = [&](int r, float x) {
    const RowStat& row = stat[r];
    const float g = logf(row.sum.h);
    const Pair e = mul(row.sum, mass(-g, mass_row(0.f, 1.f), table_h, table_l));
    const float d = x - row.top, b = d - x, de = (x - (d - b)) + (-row.top - b);
    const float h = d / t.t, l = (fmaf(-h, t.t, d) + de) / t.t;
    const Pair z = sub(Pair{h, l}, Pair{g, (e.h - 1.f) + e.l});
    return h > -INFINITY ? z.h + z.l : h;
  };
  const int32_t* drafts = after_wait(a.drafts) + static_cast<size_t>(s) * a.n;
  const float* uniform = after_wait(a.uniform) + static_cast<size_t>(s) * (a.n + 1);
  // numbers outside [0, 1) count as the nearest ones in it, a NaN as 0
  auto number = [&](int j) { return fminf(fmaxf(uniform[j], 0.f), 0x1.fffffep-1f); };
  enum { kStands, kRefused, kNoDraft, kNoTarget };
  if (tid <= a.n) {
    int what = kNoDraft;
    const RowStat p = stat[tid];
    if (!p.ok && tid <= n) {
      what = kNoTarget;
    } else if (tid < n) {
      const int x = drafts[tid];
      if (t.greedy) {
        what = p.first == x ? kStands : kRefused;
      } else {
        // u q(x) < p(x); where q(x) = 0: 0 < p(x)
        const RowStat q = lookup ? RowStat{{1.f, 0.f}, 0.f, 0, 1} : stat[a.n + 1 + tid];
        if (q.ok) {
          const float xp = logit(tid, x), xq = lookup ? q.top : logit(a.n + 1 + tid, x), u = number(tid);
          const Pair ep = mass(xp, mass_row(p.top, t.t), table_h, table_l), eq = mass(xq, mass_row(q.top, t.t), table_h, table_l);
          const Pair z = sub(mul(Pair{u, 0.f}, mul(eq, p.sum)), mul(ep, q.sum));
          const bool near = ep.h > 0x1p-60f && eq.h > 0x1p-60f && u > 0x1p-30f;
          what = (near ? z.h + z.l < 0.f : stands_far(u, xp, xq, t.t, p, q)) ? kStands : kRefused;
        }
      }
    }
    s_stands[tid] = what;
  }
  __syncthreads();
  int stop = 0;
  while (stop < a.n && s_stands[stop] == kStands) ++stop;
  const int why = s_stands[stop];
  int32_t* tokens = a.tokens + static_cast<size_t>(s) * (a.n + 1);
  float* logp = a.logp != nullptr ? a.logp + static_cast<size_t>(s) * (a.n + 1) : nullptr;
  if (cta == 0) {
    if (tid <= a.n && tid != stop) {
      tokens[tid] = tid < stop ? drafts[tid] : -1;
      if (logp != nullptr) logp[tid] = tid < stop && soft ? log_p(tid, logit(tid, drafts[tid])) : 0.f;
    }
    if (tid == 0) {
      a.accepted[s] = stop;
      if (a.lens_out != nullptr) a.lens_out[s] = max(after_wait(a.lens)[s] - (a.n - stop), 0);
      if (why == kNoTarget || t.greedy) {
        tokens[stop] = why == kNoTarget ? -1 : stat[stop].first;
        if (logp != nullptr) logp[stop] = 0.f;
      }
    }
  }
  if (why == kNoTarget || t.greedy) return;  // (the same for all CTAs of the sequence)

  const int kind = why == kNoDraft ? kFromTarget : lookup ? kWithout : kResidual;
  const T* row_p = row_of<T>(a, s, stop);
  const T* row_q = kind == kResidual ? row_of<T>(a, s, a.n + 1 + stop) : row_p;
  const int refused = kind == kFromTarget ? -1 : drafts[stop];
  const MassRow mp = mass_row(stat[stop].top, t.t);
  const MassRow mq = kind == kResidual ? mass_row(stat[a.n + 1 + stop].top, t.t) : mp;
  const Pair ratio = kind == kResidual ? div(stat[stop].sum, stat[a.n + 1 + stop].sum) : Pair{0.f, 0.f};
  // D of a token and its E_q; without a draft row p's exponential
  auto left = [&](float xp, float xq, int at, float& eq) {
    const Pair p = mass(xp, mp, table_h, table_l);
    eq = 0.f;
    if (kind != kResidual) return at == refused ? Pair{0.f, 0.f} : p;
    const Pair q = mass(xq, mq, table_h, table_l);
    eq = q.h;
    return sub(p, mul(q, ratio));
  };

  // this CTA's slice, a group of tokens per warp
  const int groups = ctas * kFinishWarps;
  VerifyGroup* sums = a.groups + static_cast<size_t>(s) * groups;
  {
    const long long g0 = (static_cast<long long>(cta) * kFinishWarps + warp) * group;
    Pair plus{0.f, 0.f}, all{0.f, 0.f};
    float b = 0.f;
    for (int i0 = 0; i0 < group; i0 += 128) {
      float xp[4], xq[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const long long at = g0 + i0 + 32 * k + lane;
        xp[k] = at < a.V ? to_f<T>(row_p[at]) : -INFINITY;
        xq[k] = kind == kResidual && at < a.V ? to_f<T>(row_q[at]) : -INFINITY;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float eq;
        const Pair d = left(xp[k], xq[k], static_cast<int>(g0) + i0 + 32 * k + lane, eq);
        const bool some = d.h + d.l > 0.f;
        add(plus, some ? d.h : 0.f, some ? d.l : 0.f);
        if (kind == kResidual) {
          add(all, d.h, d.l);
          b += some ? eq : 0.f;
        }
      }
    }
    VerifyGroup out;
    out.a = warp_sum_ll(fixed(plus, unit));
    out.d = kind == kResidual ? warp_sum_ll(fixed(all, unit)) : 0;
    out.b = warp_sum(b);
    if (lane == 0) sums[cta * kFinishWarps + warp] = out;
  }
  __threadfence();
  __syncthreads();
  if (tid == 0) {
    s_last = atomicAdd(a.done + s, 1u) == static_cast<unsigned>(ctas) - 1;
    __threadfence();
  }
  __syncthreads();
  if (!s_last) return;

  // The last CTA: k, the running sums of the groups, the group that holds the number, its token.
  // Of values in the order of the threads: the thread where the running sum, on top of
  // `offset`, first exceeds the goal (u times the whole sum where it is below 0).  Groups and
  // tokens are rounded apart: where none exceeds it, the last one with any.
  struct Pick {
    int who;  // or -1
    long long before, goal;
  };
  const float u = number(a.n);
  auto pick = [&](long long mine, long long offset, long long goal) {
    long long run = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += x;
    }
    __syncthreads();  // (what the last pick left has been read)
    if (lane == 31) s_part[warp] = run;
    __syncthreads();
    long long total = 0, base = offset;
    for (int w = 0; w < kFinishWarps; ++w) {
      if (w < warp) base += s_part[w];
      total += s_part[w];
    }
    if (goal < 0) goal = goal_of(u, total);
    const unsigned some = __ballot_sync(0xffffffffu, mine > 0);
    const unsigned above = __ballot_sync(0xffffffffu, mine > 0 && base + run > goal);
    if (lane == 0) s_first[warp] = above != 0 ? tid + __ffs(above) - 1 : -1, s_some[warp] = some != 0 ? tid + 31 - __clz(some) : -1;
    __syncthreads();
    int who = -1, last = -1;
    for (int w = kFinishWarps - 1; w >= 0; --w) {
      if (s_first[w] >= 0) who = s_first[w];
      if (last < 0) last = s_some[w];
    }
    who = who >= 0 ? who : last;
    if (tid == who) s_before = base + (run - mine);
    __syncthreads();
    return Pick{who, s_before, goal};
  };
  const int each = (groups + kFinishThreads - 1) / kFinishThreads;
  const int first = min(tid * each, groups), end = min(first + each, groups);
  long long sa = 0, sd = 0;
  float sb = 0.f;
  for (int g = first; g < end; ++g) {
    const VerifyGroup x = load_group(sums + g);
    sa += x.a, sd += x.d, sb += x.b;
  }
  float k = 0.f;
  if (kind == kResidual) {
    sd = warp_sum_ll(sd);
    if (lane == 0) s_part[warp] = sd;
    __syncthreads();
    sd = 0;
    for (int w = 0; w < kFinishWarps; ++w) sd += s_part[w];
    k = static_cast<float>(sd) / unit / stat[a.n + 1 + stop].sum.h;
  }
  Pick at = pick(max(sa - __float2ll_rn(k * sb * unit), 0ll), 0, -1);
  // nothing is left of p - q, as far as can be told: the token is drawn from p, by this CTA alone
  const bool plain = at.who < 0;
  long long lo = 0;
  int count = a.V;
  if (!plain) {
    if (tid == at.who) {
      long long before = at.before;
      for (int g = first; g < end; ++g) {
        const VerifyGroup x = load_group(sums + g);
        const long long v = x.a - __float2ll_rn(k * x.b * unit);
        if (v <= 0) continue;
        s_group = g;
        s_before = before;
        before += v;
        if (before > at.goal) break;
      }
    }
    __syncthreads();
    lo = static_cast<long long>(s_group) * group;
    count = static_cast<int>(min(static_cast<long long>(group), a.V - lo));
    at.before = s_before;
  }
  auto token_left = [&](long long i, float& x) {
    float eq;
    x = to_f<T>(row_p[i]);
    if (plain) return fixed(mass(x, mp, table_h, table_l), unit);
    Pair d = left(x, kind == kResidual ? to_f<T>(row_q[i]) : 0.f, static_cast<int>(i), eq);
    d.l -= k * eq;
    return max(fixed(d, unit), 0ll);
  };
  const int per = (count + kFinishThreads - 1) / kFinishThreads, t0 = min(tid * per, count), t1 = min(t0 + per, count);
  long long mine = 0;
  float x = 0.f;
  for (int i = t0; i < t1; ++i) mine += token_left(lo + i, x);
  at = plain ? pick(mine, 0, -1) : pick(mine, at.before, at.goal);
  if (tid == max(at.who, 0)) {
    long long before = at.before;
    int token = -1;
    float chosen = 0.f;
    for (int i = t0; i < t1; ++i) {
      const long long v = token_left(lo + i, x);
      if (v <= 0) continue;
      token = static_cast<int>(lo + i);
      chosen = x;
      before += v;
      if (before > at.goal) break;
    }
    // (a group whose sum is more than 0 only by rounding: its last token)
    if (token < 0) token = static_cast<int>(lo) + count - 1, chosen = to_f<T>(row_p[token]);
    tokens[stop] = token;
    if (logp != nullptr) logp[stop] = log_p(stop, chosen);
  }
}

template <typename T>
cudaError_t run_verify(const VerifyArgs& a, const VerifySlices& c, cudaStream_t s) {
  const int rows = a.n + 1 + (a.draft != nullptr ? a.n : 0);
  const unsigned grid = static_cast<unsigned>(a.S) * rows * a.chunks;
  ZSAA_LAUNCH(verify_scan_kernel<T>, dim3(grid), dim3(kScanThreads), 0, s, a, rows);
  int bits = 0;  // units in which sums of up to V exponentials stay below 2^62
  while ((1 << bits) < a.V) ++bits;
  ZSAA_LAUNCH(verify_finish_kernel<T>, dim3(static_cast<unsigned>(a.S) * c.ctas), dim3(kFinishThreads), 0, s, a, rows, c.ctas,
              c.group, std::ldexp(1.f, 62 - std::max(bits, 10)));
  return cudaSuccess;
}

}  // namespace

// one more than the tokens fill: a row may start inside a 16-byte block
int verify_chunks(int V) { return (V + 7 + kScanTokens - 1) / kScanTokens; }

VerifySlices verify_slices(int S, int V, int sms) {
  int group = kGroupLeast;
  auto ctas = [&] { return (V + group * kFinishWarps - 1) / (group * kFinishWarps); };
  while (group < kGroupMost && static_cast<long long>(S) * ctas() > 4 * sms) group *= 2;
  return VerifySlices{ctas(), group};
}
int verify_groups_most(int V) { return (V + kGroupLeast * kFinishWarps - 1) / (kGroupLeast * kFinishWarps) * kFinishWarps; }

cudaError_t launch_draft_verify(const VerifyArgs& a, int dtype, int sms, cudaStream_t s) {
  const VerifySlices c = verify_slices(a.S, a.V, sms);
  return dtype == ZSAA_F32 ? run_verify<float>(a, c, s) : run_verify<bf16>(a, c, s);
}

}  // namespace zsaa
