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
constexpr float kLn2H = 0.693147182464599609375f;  // ln 2 rounded to float, and what that leaves
constexpr float kLn2L = static_cast<float>(0.69314718055994530942 - static_cast<double>(kLn2H));

__device__ __forceinline__ Pair mass(float x, const MassRow& r, const float* table_h, const float* table_l) {
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

// The same of two tokens at once, in packed arithmetic (whose products are never fused into
// what follows).  Negated products come from negated factors.
struct Pair2 {
  uint64_t h, l;
};
struct MassRow2 {
  uint64_t m, nm, ch, nch, cl;
};
__device__ __forceinline__ uint64_t both(float x) { return f2pack(x, x); }
__device__ __forceinline__ MassRow2 mass_row2(const MassRow& r) {
  return MassRow2{both(r.m), both(-r.m), both(r.ch), both(-r.ch), both(r.cl)};
}
__device__ __forceinline__ Pair2 mass2(float x0, float x1, const MassRow2& r, const float* table_h, const float* table_l) {
  const uint64_t x = f2pack(x0, x1);
  const uint64_t d = fsub2(x, r.m), b = fsub2(d, x);
  const uint64_t de = fadd2(fsub2(x, fsub2(d, b)), fsub2(r.nm, b));
  const uint64_t ny = fmul2(d, r.nch);
  const uint64_t ye = fadd2(ffma2(d, r.ch, ny), ffma2(d, r.cl, fmul2(de, r.ch)));
  const uint64_t magic = ffma2(ny, both(-32.f), both(0x1.8p23f));
  const uint64_t nf = ffma2(fsub2(magic, both(0x1.8p23f)), both(0.03125f), ny);
  const uint64_t g = fmul2(nf, both(-kLn2H)), ng = fmul2(nf, both(kLn2H));
  const uint64_t ge = fadd2(ffma2(nf, both(-kLn2H), ng), ffma2(nf, both(-kLn2L), fmul2(ye, both(kLn2H))));
  const uint64_t w = fadd2(g, ge);
  const uint64_t rest = ffma2(fmul2(w, w), ffma2(w, ffma2(w, both(1.f / 24.f), both(1.f / 6.f)), both(0.5f)), ge);
  float magic0, magic1, ny0, ny1;
  f2unpack(magic, magic0, magic1);
  f2unpack(ny, ny0, ny1);
  const int k0 = __float_as_int(magic0) - __float_as_int(0x1.8p23f), k1 = __float_as_int(magic1) - __float_as_int(0x1.8p23f);
  const uint64_t th = f2pack(table_h[k0 & 31], table_h[k1 & 31]), tl = f2pack(table_l[k0 & 31], table_l[k1 & 31]);
  const uint64_t ph = fmul2(th, g), nph = fmul2(th, ng);
  const uint64_t pl = fadd2(ffma2(th, g, nph), ffma2(th, rest, ffma2(tl, g, tl)));
  const uint64_t h = fadd2(th, ph), l = fadd2(fsub2(ph, fsub2(h, th)), pl);
  // (2^(k/32 whole) where y > -125; elsewhere whatever it is, it is not taken)
  const uint64_t scale = f2pack(__int_as_float(((k0 & ~31) << 18) + 0x3f800000), __int_as_float(((k1 & ~31) << 18) + 0x3f800000));
  float h0, h1, l0, l1;
  f2unpack(fmul2(h, scale), h0, h1);
  f2unpack(fmul2(l, scale), l0, l1);
  return Pair2{f2pack(ny0 < 125.f ? h0 : 0.f, ny1 < 125.f ? h1 : 0.f), f2pack(ny0 < 125.f ? l0 : 0.f, ny1 < 125.f ? l1 : 0.f)};
}
__device__ __forceinline__ void add2(Pair2& s, uint64_t h, uint64_t l) {
  const uint64_t t = fadd2(s.h, h), b = fsub2(t, s.h);
  s.l = fadd2(s.l, fadd2(fadd2(fsub2(s.h, fsub2(t, b)), fsub2(h, b)), l));
  s.h = t;
}
// a - c b with the pair c (nh, l: its negated first part and its second)
__device__ __forceinline__ Pair2 less2(const Pair2& a, const Pair2& b, uint64_t ch, uint64_t nch, uint64_t cl) {
  const uint64_t nh = fmul2(b.h, nch), e = ffma2(b.h, ch, nh);  // -(b c) and what rounding took off
  const uint64_t cb = fadd2(e, ffma2(b.h, cl, fmul2(b.l, ch)));
  const uint64_t h = fadd2(a.h, nh), c = fsub2(h, a.h);
  return Pair2{h, fadd2(fadd2(fsub2(a.h, fsub2(h, c)), fsub2(nh, c)), fsub2(a.l, cb))};
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
constexpr int kFinishPerSm = 3;
constexpr int kGroupStep = 128;    // a group, the tokens of a warp, is a multiple of it
constexpr int kGroupsMost = 1024;  // groups of a sequence, at most

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
__global__ void __launch_bounds__(kFinishThreads, kFinishPerSm)
    verify_finish_kernel(const __grid_constant__ VerifyArgs a, int rows, int ctas, int group, float unit) {
  __shared__ float table_h[32], table_l[32];
  __shared__ RowStat stat[2 * kVerifyMaxDrafts + 1];
  __shared__ int s_stop, s_why;
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
  // one round trip: temperature, drafts, numbers, the rows' stretches; then the drafts' logits
  const Temperature t = temperature_of(a, s);
  const int n = drafts_of(a, s);
  const bool lookup = a.draft == nullptr, soft = !t.greedy && !t.bad;
  const int32_t* drafts = after_wait(a.drafts) + static_cast<size_t>(s) * a.n;
  const float* uniform = after_wait(a.uniform) + static_cast<size_t>(s) * (a.n + 1);
  // numbers outside [0, 1) count as the nearest ones in it, a NaN as 0
  auto number = [&](int j) { return fminf(fmaxf(uniform[j], 0.f), 0x1.fffffep-1f); };
  auto logit = [&](int r, int x) { return to_f<T>(row_of<T>(a, s, r)[x]); };
  const float u = number(a.n);
  float my_u = 0.f, xp = 0.f, xq = 0.f;
  int my_draft = -1;
  if (tid < n) {
    my_draft = drafts[tid];
    my_u = number(tid);
    xp = logit(tid, my_draft);
    if (!lookup && soft) xq = logit(a.n + 1 + tid, my_draft);
  }
  const int4* chunks = after_wait(reinterpret_cast<const int4*>(a.stat)) + static_cast<size_t>(s) * rows * a.chunks;
  auto chunk_at = [&](int r, int i) {
    const int4 v = chunks[static_cast<size_t>(r) * a.chunks + i];
    VerifyChunk c;
    c.sum = static_cast<long long>(static_cast<unsigned long long>(static_cast<unsigned>(v.y)) << 32 | static_cast<unsigned>(v.x));
    c.top = __int_as_float(v.z);
    c.first = v.w;
    return c;
  };

  // every row's maximum and sum, of 16 or 32 lanes (rows that the scan left out: anything)
  const int lanes = a.chunks <= 16 ? 16 : 32, per_warp = 32 / lanes;
  for (int r0 = warp * per_warp; r0 < rows; r0 += kFinishWarps * per_warp) {
    const int r = min(r0 + lane / lanes, rows - 1), l = lane & (lanes - 1);
    float top = -INFINITY;
    int bad = 0;
    for (int i = l; i < a.chunks; i += lanes) {
      const VerifyChunk c = chunk_at(r, i);
      top = fmaxf(top, c.top);
      bad |= c.first < 0;
    }
    for (int o = lanes / 2; o > 0; o >>= 1) {
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      bad |= __shfl_xor_sync(0xffffffffu, bad, o);
    }
    Pair sum{0.f, 0.f};
    int first = a.V;
    const MassRow m = mass_row(top, t.t);
    for (int i = l; i < a.chunks; i += lanes) {
      const VerifyChunk c = chunk_at(r, i);
      if (t.greedy) {
        if (c.top == top) first = min(first, c.first);
      } else {
        const Pair v = mul(pair_of(c.sum, 1.f / kSumScale), mass(c.top, m, table_h, table_l));
        if (c.top > -INFINITY) add(sum, v.h, v.l);
      }
    }
    for (int o = lanes / 2; o > 0; o >>= 1) {
      const float h = __shfl_xor_sync(0xffffffffu, sum.h, o), e = __shfl_xor_sync(0xffffffffu, sum.l, o);
      add(sum, h, e);
      first = min(first, __shfl_xor_sync(0xffffffffu, first, o));
    }
    if (l == 0 && r0 + lane / lanes < rows) stat[r] = RowStat{sum, top, first, !t.bad && bad == 0 && top > -INFINITY};
  }
  __syncthreads();
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
  enum { kStands, kRefused, kNoDraft, kNoTarget };
  if (warp == 0) {  // (lane j: draft j)
    int what = kNoDraft;
    const RowStat p = stat[min(lane, a.n)];
    if (!p.ok) {
      what = kNoTarget;
    } else if (lane < n) {
      if (t.greedy) {
        what = p.first == my_draft ? kStands : kRefused;
      } else {
        // u q(x) < p(x); where q(x) = 0: 0 < p(x)
        const RowStat q = lookup ? RowStat{{1.f, 0.f}, 0.f, 0, 1} : stat[a.n + 1 + lane];
        if (q.ok) {
          const Pair ep = mass(xp, mass_row(p.top, t.t), table_h, table_l), eq = mass(xq, mass_row(q.top, t.t), table_h, table_l);
          const Pair z = sub(mul(Pair{my_u, 0.f}, mul(eq, p.sum)), mul(ep, q.sum));
          const bool near = ep.h > 0x1p-60f && eq.h > 0x1p-60f && my_u > 0x1p-30f;
          what = (near ? z.h + z.l < 0.f : stands_far(my_u, xp, xq, t.t, p, q)) ? kStands : kRefused;
        }
      }
    }
    const int stop = __ffs(__ballot_sync(0xffffffffu, what != kStands || lane >= a.n)) - 1;
    what = __shfl_sync(0xffffffffu, what, stop);
    if (lane == 0) s_stop = stop, s_why = what;
  }
  __syncthreads();
  const int stop = s_stop, why = s_why;
  int32_t* tokens = a.tokens + static_cast<size_t>(s) * (a.n + 1);
  float* logp = a.logp != nullptr ? a.logp + static_cast<size_t>(s) * (a.n + 1) : nullptr;
  if (cta == 0) {
    if (tid <= a.n && tid != stop) {
      tokens[tid] = tid < stop ? my_draft : -1;
      if (logp != nullptr) logp[tid] = tid < stop && soft ? log_p(tid, xp) : 0.f;
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

  // this CTA's slice, a group of tokens per warp
  const int groups = ctas * kFinishWarps;
  VerifyGroup* sums = a.groups + static_cast<size_t>(s) * groups;
  {
    const long long g0 = (static_cast<long long>(cta) * kFinishWarps + warp) * group;
    const MassRow2 p2 = mass_row2(mp);
    Pair2 plus{0, 0}, all{0, 0};
    float b = 0.f;
    auto load = [&](const T* row, int i0, float (&x)[4]) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const long long at = g0 + i0 + 32 * k + lane;
        x[k] = i0 < group && at < a.V ? to_f<T>(row[at]) : -INFINITY;
      }
    };
    float x[4], next[4];
    load(row_p, 0, x);
    if (kind == kResidual) {
      const MassRow2 q2 = mass_row2(mq);
      const uint64_t ch = both(ratio.h), nch = both(-ratio.h), cl = both(ratio.l);
      float y[4], next_y[4];
      load(row_q, 0, y);
      for (int i0 = 0; i0 < group; i0 += 128) {
        load(row_p, i0 + 128, next);
        load(row_q, i0 + 128, next_y);
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
          const Pair2 q = mass2(y[k], y[k + 1], q2, table_h, table_l);
          const Pair2 d = less2(mass2(x[k], x[k + 1], p2, table_h, table_l), q, ch, nch, cl);
          add2(all, d.h, d.l);
          float s0, s1, h0, h1, l0, l1, q0, q1;
          f2unpack(fadd2(d.h, d.l), s0, s1);
          f2unpack(d.h, h0, h1);
          f2unpack(d.l, l0, l1);
          f2unpack(q.h, q0, q1);
          add2(plus, f2pack(s0 > 0.f ? h0 : 0.f, s1 > 0.f ? h1 : 0.f), f2pack(s0 > 0.f ? l0 : 0.f, s1 > 0.f ? l1 : 0.f));
          b += (s0 > 0.f ? q0 : 0.f) + (s1 > 0.f ? q1 : 0.f);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = next[k], y[k] = next_y[k];
      }
    } else {
      for (int i0 = 0; i0 < group; i0 += 128) {
        load(row_p, i0 + 128, next);
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
          const long long at = g0 + i0 + 32 * k + lane;
          const Pair2 p = mass2(at == refused ? -INFINITY : x[k], at + 32 == refused ? -INFINITY : x[k + 1], p2, table_h, table_l);
          add2(plus, p.h, p.l);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = next[k];
      }
    }
    // the two tokens' sums, in units
    auto joined = [&](const Pair2& v) {
      float h0, h1, l0, l1;
      f2unpack(v.h, h0, h1);
      f2unpack(v.l, l0, l1);
      return warp_sum_ll(fixed(Pair{h0, l0}, unit) + fixed(Pair{h1, l1}, unit));
    };
    VerifyGroup out;
    out.a = joined(plus);
    out.d = kind == kResidual ? joined(all) : 0;
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
#pragma unroll
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
#pragma unroll
    for (int w = kFinishWarps - 1; w >= 0; --w) {
      if (s_first[w] >= 0) who = s_first[w];
      if (last < 0) last = s_some[w];
    }
    who = who >= 0 ? who : last;
    if (tid == who) s_before = base + (run - mine);
    __syncthreads();
    return Pick{who, s_before, goal};
  };
  constexpr int EACH = kGroupsMost / kFinishThreads;  // groups of a thread
  const int each = (groups + kFinishThreads - 1) / kFinishThreads, g0 = tid * each;
  VerifyGroup mine_g[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    mine_g[i] = VerifyGroup{0, 0, 0.f};
    if (i < each && g0 + i < groups) mine_g[i] = load_group(sums + g0 + i);
  }
  float k = 0.f;
  if (kind == kResidual) {
    long long sd = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) sd += mine_g[i].d;
    sd = warp_sum_ll(sd);
    if (lane == 0) s_part[warp] = sd;
    __syncthreads();
    sd = 0;
#pragma unroll
    for (int w = 0; w < kFinishWarps; ++w) sd += s_part[w];
    k = static_cast<float>(sd) / unit / stat[a.n + 1 + stop].sum.h;
  }
  long long mine = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    mine_g[i].a = max(mine_g[i].a - __float2ll_rn(k * mine_g[i].b * unit), 0ll);
    mine += mine_g[i].a;
  }
  Pick at = pick(mine, 0, -1);
  // nothing is left of p - q, as far as can be told: the token is drawn from p, by this CTA alone
  const bool plain = at.who < 0;
  long long lo = 0;
  int count = a.V;
  if (!plain) {
    if (tid == at.who) {
      long long before = at.before;
      bool found = false;
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        if (found || mine_g[i].a == 0) continue;
        s_group = g0 + i;
        s_before = before;
        before += mine_g[i].a;
        found = before > at.goal;
      }
    }
    __syncthreads();
    lo = static_cast<long long>(s_group) * group;
    count = static_cast<int>(min(static_cast<long long>(group), a.V - lo));
    at.before = s_before;
  }
  // a token's share of the sum
  auto token_left = [&](long long i, float& x) {
    x = to_f<T>(row_p[i]);
    const Pair p = mass(x, mp, table_h, table_l);
    if (plain || kind != kResidual) return !plain && i == refused ? 0ll : fixed(p, unit);
    const Pair q = mass(to_f<T>(row_q[i]), mq, table_h, table_l);
    Pair d = sub(p, mul(q, ratio));
    d.l -= k * q.h;
    return max(fixed(d, unit), 0ll);
  };
  const int per = (count + kFinishThreads - 1) / kFinishThreads, t0 = min(tid * per, count), t1 = min(t0 + per, count);
  mine = 0;
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

// CTAs of a sequence: as many as there are at once for it, each with 128 tokens a warp or more.
static VerifySlices verify_slices(int V, long long at_once) {
  const int tokens = kGroupStep * kFinishWarps, most = std::min((V + tokens - 1) / tokens, kGroupsMost / kFinishWarps);
  const int ctas = static_cast<int>(std::max(1ll, std::min(static_cast<long long>(most), at_once)));
  const int group = ((V + ctas * kFinishWarps - 1) / (ctas * kFinishWarps) + kGroupStep - 1) / kGroupStep * kGroupStep;
  return VerifySlices{(V + group * kFinishWarps - 1) / (group * kFinishWarps), group};
}
int verify_groups_most(int V) { return verify_slices(V, kGroupsMost).ctas * kFinishWarps; }

cudaError_t launch_draft_verify(const VerifyArgs& a, int dtype, int sms, cudaStream_t s) {
  const VerifySlices c = verify_slices(a.V, kFinishPerSm * sms / a.S);
  return dtype == ZSAA_F32 ? run_verify<float>(a, c, s) : run_verify<bf16>(a, c, s);
}

}  // namespace zsaa
