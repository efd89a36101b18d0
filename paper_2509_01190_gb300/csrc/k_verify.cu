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
//                         exponentials.  Bound by the logits' bytes (64 sequences of 5 drafts over
//                         128256 float32 logits: 57 us, 5.8 TB/s).
//   verify_finish_kernel  the rows at which a sequence stops again, a group of tokens per CTA;
//                         a sequence's last CTA finds the token.  Bound by its chain of round trips
//                         on few sequences (9 us of the 14 that one of 4 drafts takes), by the FMA
//                         pipe on many (the same 64: 41 us, half of it with that pipe busy).
//
// Small calls scan all rows at once, and every CTA of the second kernel works out which drafts
// stand.  Large calls scan draft 0's rows of all sequences first, then draft 1's, and so on
// (verify_scan_in_turn_kernel, behind verify_start_kernel); the CTA that ends a draft's rows decides
// it, and rows behind a refused draft, which nothing depends on, are left out as far as that is
// known when their turn comes.
//
// What decides a draft is one comparison of two quotients, off by some 1e-7 with sums of
// float32 exponentials: a sum is off by 4e-8 as a rule and 1.6e-7 at most over rows of 128256
// logits (normal ones of deviation 0.01, 3 and 30, and ones that fall as the logarithm of their
// rank) at temperatures from 0.05 to 10, much of it log2(e) / T as one float; and by less than 2^-17
// on any row (three roundings of an exponential's argument, its own 2^-22, the additions).
// What decides a token is where u_n falls among V borders, some 1e-5 apart and closer: a running
// sum that is off by 1e-9 picks the wrong token every few thousand calls.  So the rows at which
// a sequence stops are gone through again with exponentials as pairs of floats, good to 2^-35.7
// each and without a bias to see (below 2^-42), and sums in pairs and in 64-bit integers.
//
// One pass does it, although the residual needs the sums of both rows: with E the exponentials,
// Z their exact sums and c0 the quotient Z_p / Z_q as the scan has it, the pass adds up
//   D_i = E_p,i - c0 E_q,i        over all tokens, and
//   A = sum D_i, B = sum E_q,i    over a group's tokens with D_i > 0.
// The exact quotient is c0 + k with k = sum D / Z_q, some 2^-21 of it (2^-16 at most), so a group's
// residual is A - k B.  A token whose D_i changes its sign with k is off by k E_q,i at most, and such
// tokens' quotients all lie within 2^-21 of Z_p / Z_q: as small a part of the mass, as a rule.  (Where
// they may not be, choose_alone goes through the tokens again.)
// (Two passes, the first for the sums, took 270 us on the 64 where this one took 77, both still with
// sums of 64-bit floats.)
//
// 64-bit floats are left out of the sums: the SM does two of their operations a clock.
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

// drafts of sequence s before the first that is no token (whole warps)
__device__ __forceinline__ int drafts_of(const VerifyArgs& a, int s) {
  const int lane = threadIdx.x & 31;
  const int x = lane < a.n ? after_wait(a.drafts)[static_cast<size_t>(s) * a.n + lane] : -1;
  return __ffs(__ballot_sync(0xffffffffu, x < 0 || x >= a.V)) - 1;  // (lane 31 has no draft)
}

// 32 values of a thread as they are stored, 16 bytes to a vector.
constexpr int kScanValues = 32;
template <typename T>
struct Stored {
  static constexpr int VEC = 16 / sizeof(T);
  uint4 v[kScanValues / VEC];
  __device__ __forceinline__ float at(int k) const {
    const uint4& u = v[k / VEC];
    if constexpr (sizeof(T) == 2) {
      const uint32_t w = k % VEC < 2 ? u.x : k % VEC < 4 ? u.y : k % VEC < 6 ? u.z : u.w;
      return k % 2 == 0 ? bf16lo(w) : bf16hi(w);
    } else {
      return __uint_as_float(k % VEC == 0 ? u.x : k % VEC == 1 ? u.y : k % VEC == 2 ? u.z : u.w);
    }
  }
};
__device__ __forceinline__ uint32_t bits_of(float x) { return __float_as_uint(x); }
__device__ __forceinline__ uint32_t bits_of(bf16 x) { return __bfloat16_as_ushort(x); }

// Row r of sequence s: target row r for r <= n, else draft row r - n - 1.
template <typename T>
__device__ __forceinline__ const T* row_of(const VerifyArgs& a, int s, int r) {
  if (r <= a.n) return after_wait(static_cast<const T*>(a.target)) + (static_cast<long long>(s) * (a.n + 1) + r) * a.ld;
  return after_wait(static_cast<const T*>(a.draft)) + (static_cast<long long>(s) * a.n + (r - a.n - 1)) * a.draft_ld;
}

constexpr float kSumScale = 0x1p36f;  // a stretch's sum, at most 2^13, in units of 2^-36

// ---------------------------------------------------------------- exponentials as pairs of floats

struct Pair {
  float h, l;
};

// 2^(i/32) as pairs of floats: all first parts, then the second parts relative to the first
struct Powers {
  float v[64];
};
constexpr Powers powers() {
  Powers p{};
  double x = 1.0;
  for (int i = 0; i < 32; ++i) {
    p.v[i] = static_cast<float>(x);
    p.v[32 + i] = static_cast<float>((x - static_cast<double>(p.v[i])) / static_cast<double>(p.v[i]));
    x *= 1.02189714865411667823;  // 2^(1/32)
  }
  return p;
}
__constant__ Powers kPowers = powers();

// exp((x - m) / T) = 2^y: y = (x - m) log2(e) / T with its rounding errors kept, cut into
// k / 32 and a rest f of at most 1/64; 2^(k/32) from a table of pairs, 2^f by its series, whose
// first term is a pair too (|f ln 2| <= 0.0109: the terms from the second on are below 2^-14 and
// their float32 errors below 2^-37, as is the first one left out).  0 below 2^-125.  Off by at most
// 2^-35.7 over 9.6 million values at temperatures from 0.05 to 60 and logits up to 1e6.
//
// m is not the row's maximum but the next multiple above it of a power of two s <= T / log2(e)
// (the maximum itself where that is one of s / 2): with d = x - m rounded, d + m and x - (d + m)
// are then exact wherever 2^y counts.  For |d| <= 250 s, so m is a multiple of d's last place; d + m
// is one too and no larger than x and half a place, of which d + m differs from x only where x
// has finer places than d, so it fits a float; and x - (d + m) are low places of x.
struct MassRow {
  float m, ch, cl;  // m; log2(e) / T
};
__device__ __forceinline__ MassRow mass_row(float t) {  // without its m
  constexpr float kLog2eH = 1.44269502162933349609375f;
  constexpr float kLog2eL = static_cast<float>(1.4426950408889634074 - static_cast<double>(kLog2eH));
  const float ch = kLog2eH / t;
  return MassRow{0.f, ch, (fmaf(-ch, t, kLog2eH) + kLog2eL) / t};
}
__device__ __forceinline__ MassRow row_at(MassRow r, float m) {
  r.m = m;
  return r;
}
__device__ __forceinline__ MassRow row_above(MassRow r, float top) {  // of a row with the maximum `top`
  const int e = ilogbf(r.ch) + 1;  // ch < 2^e: s = 2^-e
  r.m = fabsf(top) < ldexpf(1.f, 22 - e) ? ldexpf(ceilf(ldexpf(top, e)), -e) : top;
  return r;
}
constexpr float kLn2H = 0.693147182464599609375f;  // ln 2 rounded to float, and what that leaves
constexpr float kLn2L = static_cast<float>(0.69314718055994530942 - static_cast<double>(kLn2H));

__device__ __forceinline__ Pair mass(float x, const MassRow& r, const float* table) {
  const float d = x - r.m, de = x - (d + r.m);  // what rounding took off x - m
  const float y = __fmul_rn(d, r.ch);  // (products whose rounding is kept are not fused into what follows)
  const float ye = fmaf(d, r.cl, fmaf(de, r.ch, fmaf(d, r.ch, -y)));
  const float magic = fmaf(y, 32.f, 0x1.8p23f);
  const int k = __float_as_int(magic) - __float_as_int(0x1.8p23f);
  const float f = fmaf(magic - 0x1.8p23f, -0.03125f, y);
  const float g = __fmul_rn(f, kLn2H);
  const float ge = fmaf(ye, kLn2H, fmaf(f, kLn2L, fmaf(f, kLn2H, -g)));
  const float w = g + ge, tl = table[32 + (k & 31)];
  const float rest = fmaf(tl, g, fmaf(w * w, fmaf(w, fmaf(w, 1.f / 24.f, 1.f / 6.f), 0.5f), ge)) + tl;
  const float th = __int_as_float(__float_as_int(table[k & 31]) + ((k & ~31) << 18));  // times 2^(k/32 whole)
  const float ph = __fmul_rn(th, g);
  const float pl = fmaf(th, rest, fmaf(th, g, -ph));
  const float h = th + ph, l = (ph - (h - th)) + pl;
  return y > -125.f ? Pair{h, l} : Pair{0.f, 0.f};
}

// The same of two tokens at once, in packed arithmetic (whose products are never fused into
// what follows).
struct Pair2 {
  uint64_t h, l;
};
struct Factor2 {
  uint64_t ch, nch, cl;
};
__device__ __forceinline__ uint64_t both(float x) { return f2pack(x, x); }
__device__ __forceinline__ uint64_t negated(uint64_t x) { return x ^ 0x8000000080000000ull; }
__device__ __forceinline__ Factor2 factor2(const MassRow& r) { return Factor2{both(r.ch), both(-r.ch), both(r.cl)}; }
__device__ __forceinline__ Pair2 mass2(float x0, float x1, uint64_t m, const Factor2& r, const float* table) {
  const uint64_t x = f2pack(x0, x1);
  const uint64_t d = fsub2(x, m), de = fsub2(x, fadd2(d, m));
  const uint64_t ny = fmul2(d, r.nch);
  const uint64_t ye = ffma2(d, r.cl, ffma2(de, r.ch, ffma2(d, r.ch, ny)));
  const uint64_t magic = ffma2(ny, both(-32.f), both(0x1.8p23f));
  const uint64_t nf = ffma2(fsub2(magic, both(0x1.8p23f)), both(0.03125f), ny);
  const uint64_t ng = fmul2(nf, both(kLn2H)), g = negated(ng);
  const uint64_t ge = ffma2(ye, both(kLn2H), ffma2(nf, both(-kLn2L), ffma2(nf, both(-kLn2H), ng)));
  const uint64_t w = fadd2(g, ge);
  float magic0, magic1, ny0, ny1;
  f2unpack(magic, magic0, magic1);
  f2unpack(ny, ny0, ny1);
  const int k0 = __float_as_int(magic0) - __float_as_int(0x1.8p23f), k1 = __float_as_int(magic1) - __float_as_int(0x1.8p23f);
  const uint64_t tl = f2pack(table[32 + (k0 & 31)], table[32 + (k1 & 31)]);
  const uint64_t th = f2pack(__int_as_float(__float_as_int(table[k0 & 31]) + ((k0 & ~31) << 18)),
                             __int_as_float(__float_as_int(table[k1 & 31]) + ((k1 & ~31) << 18)));
  const uint64_t series = ffma2(fmul2(w, w), ffma2(w, ffma2(w, both(1.f / 24.f), both(1.f / 6.f)), both(0.5f)), ge);
  const uint64_t rest = fadd2(ffma2(tl, g, series), tl);
  const uint64_t ph = fmul2(th, g);
  const uint64_t pl = ffma2(th, rest, ffma2(th, g, negated(ph)));
  const uint64_t h = fadd2(th, ph), l = fadd2(fsub2(ph, fsub2(h, th)), pl);
  float h0, h1, l0, l1;
  f2unpack(h, h0, h1);
  f2unpack(l, l0, l1);
  // (where y is not above -125 they are whatever they are)
  return Pair2{f2pack(ny0 < 125.f ? h0 : 0.f, ny1 < 125.f ? h1 : 0.f), f2pack(ny0 < 125.f ? l0 : 0.f, ny1 < 125.f ? l1 : 0.f)};
}
// to a sum whose first part is never smaller than h
__device__ __forceinline__ void add_below2(Pair2& s, uint64_t h, uint64_t l) {
  const uint64_t t = fadd2(s.h, h);
  s.l = fadd2(s.l, fadd2(fsub2(h, fsub2(t, s.h)), l));
  s.h = t;
}
// a - c b with the pair c (nh, l: its negated first part and its second)
__device__ __forceinline__ Pair2 less2(const Pair2& a, const Pair2& b, uint64_t ch, uint64_t nch, uint64_t cl) {
  const uint64_t nh = fmul2(b.h, nch), e = ffma2(b.h, ch, nh);  // -(b c) and what rounding took off
  const uint64_t cb = ffma2(b.l, ch, ffma2(b.h, cl, e));
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

// Adds to a count on the device, ordered after what the warp has stored (and __syncwarp) and before
// what it loads from L2; returns the old count.
__device__ __forceinline__ unsigned add_acq_rel(unsigned* p, unsigned v) {
  unsigned old;
  asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], %2;" : "=r"(old) : "l"(p), "r"(v) : "memory");
  return old;
}

// ---------------------------------------------------------------- decisions

enum { kStands, kRefused, kNoDraft, kNoTarget };

// u q(x) < p(x) from the logits alone, where the exponentials are too small for float pairs
__device__ __noinline__ bool stands_far(float u, float xp, float xq, float t, const VerifyRow& p, const VerifyRow& q,
                                        bool lookup) {
  auto log_of = [t](float x, const VerifyRow& r) {
    const double sum = static_cast<double>(r.sum_h) + static_cast<double>(r.sum_l);
    return (static_cast<double>(x) - static_cast<double>(r.m)) / t - log(sum);
  };
  const double lp = log_of(xp, p), lq = lookup ? 0.0 : log_of(xq, q);
  // (u = 0: wherever p(x) > 0, however small; the quotient may be below the least number above 0)
  return lp > -INFINITY && (lq == -INFINITY || u == 0.f || u < exp(lp - lq));
}

// What a sequence's rows have in common.
struct Sequence {
  Temperature t;
  MassRow factor;
  bool soft, lookup;  // a temperature above 0; no draft rows
  int n;              // drafts before the first that is no token
};
__device__ __forceinline__ Sequence sequence_with(const VerifyArgs& a, const Temperature& t, int n) {
  return Sequence{t, mass_row(t.t), !t.greedy && !t.bad, a.draft == nullptr, n};
}
// numbers outside [0, 1) count as the nearest ones in it, a NaN as 0
__device__ __forceinline__ float number_at(const VerifyArgs& a, int s, int j) {
  return fminf(fmaxf(after_wait(a.uniform)[static_cast<size_t>(s) * (a.n + 1) + j], 0.f), 0x1.fffffep-1f);
}
template <typename T>
__device__ __forceinline__ float logit_at(const VerifyArgs& a, int s, int r, int x) {
  return to_f<T>(row_of<T>(a, s, r)[x]);
}

// What becomes of draft j < q.n (or kNoDraft, kNoTarget), with the logits of its token.
__device__ __forceinline__ int verdict(const Sequence& q, int j, int draft, float u, float xp, float xq, const VerifyRow& p,
                                       const VerifyRow& draft_row, const float* table) {
  if (!p.ok) return kNoTarget;
  if (j >= q.n) return kNoDraft;
  if (q.t.greedy) return p.first == draft ? kStands : kRefused;
  if (!q.lookup && !draft_row.ok) return kNoDraft;
  // u q(x) < p(x); where q(x) = 0: 0 < p(x)
  const Pair one{1.f, 0.f}, ep = mass(xp, row_at(q.factor, p.m), table);
  const Pair eq = q.lookup ? one : mass(xq, row_at(q.factor, draft_row.m), table);
  const Pair zq = q.lookup ? one : Pair{draft_row.sum_h, draft_row.sum_l};
  const Pair z = sub(mul(Pair{u, 0.f}, mul(eq, Pair{p.sum_h, p.sum_l})), mul(ep, zq));
  const bool near = ep.h > 0x1p-60f && eq.h > 0x1p-60f && u > 0x1p-30f;
  return (near ? z.h + z.l < 0.f : stands_far(u, xp, xq, q.t.t, p, draft_row, q.lookup)) ? kStands : kRefused;
}

__device__ __forceinline__ VerifyChunk load_chunk(const VerifyChunk* p) {
  const int4 v = __ldcg(reinterpret_cast<const int4*>(p));
  VerifyChunk c;
  c.sum = static_cast<long long>(static_cast<uint64_t>(static_cast<uint32_t>(v.y)) << 32 | static_cast<uint32_t>(v.x));
  c.top = __int_as_float(v.z);
  c.first = v.w;
  return c;
}

// A row from its n stretches, by `lanes` lanes (16 or 32) of a warp, the same in all of them.  mine: the
// stretch of this lane's number, where there is one.
__device__ __forceinline__ VerifyRow row_total(const VerifyChunk* chunks, VerifyChunk mine, int n, int lanes,
                                               const Sequence& q, int V, const float* table) {
  const int l = threadIdx.x & (lanes - 1);
  auto chunk_at = [&](int i) { return load_chunk(chunks + i); };
  if (l >= n) mine = VerifyChunk{0, -INFINITY, V};
  float top = mine.top;
  int bad = mine.first < 0;
  for (int i = l + lanes; i < n; i += lanes) {
    const VerifyChunk c = chunk_at(i);
    top = fmaxf(top, c.top);
    bad |= c.first < 0;
  }
  for (int o = lanes / 2; o > 0; o >>= 1) {
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    bad |= __shfl_xor_sync(0xffffffffu, bad, o);
  }
  Pair sum{0.f, 0.f};
  int first = V;
  const MassRow m = row_above(q.factor, top);
  for (int i = l; i < n; i += lanes) {
    const VerifyChunk c = i == l ? mine : chunk_at(i);
    if (q.t.greedy) {
      if (c.top == top) first = min(first, c.first);
    } else {
      const Pair v = mul(pair_of(c.sum, 1.f / kSumScale), mass(c.top, m, table));
      if (c.top > -INFINITY) add(sum, v.h, v.l);
    }
  }
  for (int o = lanes / 2; o > 0; o >>= 1) {
    const float h = __shfl_xor_sync(0xffffffffu, sum.h, o), e = __shfl_xor_sync(0xffffffffu, sum.l, o);
    add(sum, h, e);
    first = min(first, __shfl_xor_sync(0xffffffffu, first, o));
  }
  return VerifyRow{sum.h, sum.l, m.m, first, !q.t.bad && bad == 0 && top > -INFINITY};
}

// ---------------------------------------------------------------- the rows' maxima and sums

// CTAs to an SM, for the scan of all rows and for the one in turn.  Threads keep their logits as they
// are stored, so bf16 takes half the registers (us, 24 sequences of 3 drafts over 50257 bf16 logits:
// unpacked, 4 to an SM 19.2, packed 4 18.8, 5 18.5, 6 18.9; in turn, 64 of 5 over 128256: 3 62.9,
// 4 60.0, 5 62.0).
template <typename T>
constexpr int kScanPerSm = sizeof(T) == 2 ? 5 : 4;
template <typename T>
constexpr int kTurnPerSm = sizeof(T) == 2 ? 4 : 3;
constexpr int kScanThreads = 256, kScanTokens = kScanThreads * kScanValues;

// Sum over the warp of values in [0, 2^50) (two 32-bit reductions of 25 bits each).
__device__ __forceinline__ unsigned long long warp_sum_u50(unsigned long long v) {
  const unsigned lo = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(v) & 0x1ffffffu);
  const unsigned hi = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(v >> 25));
  return (static_cast<unsigned long long>(hi) << 25) + lo;
}

// One stretch of a row.  Every warp takes its sum against its own maximum, so the warps meet
// once; warp 0 then has the stretch.
struct StretchParts {
  float top[kScanThreads / 32];
  unsigned long long sum[kScanThreads / 32];
  int first[kScanThreads / 32];
};
template <typename T>
__device__ __forceinline__ void load_stretch(const T* row, int chunk, int V, Stored<T>& x) {
  constexpr int VEC = Stored<T>::VEC, PER_WORD = 4 / sizeof(T);
  // the stretch starts on a 16-byte boundary, before the row's first token for the first one
  const int lead = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
  const int t0 = chunk * kScanTokens - lead;
#pragma unroll
  for (int k = 0; k < kScanValues / VEC; ++k) {
    const int at = t0 + (k * kScanThreads + static_cast<int>(threadIdx.x)) * VEC;
    if (at >= 0 && at <= V - VEC) {
      x.v[k] = *reinterpret_cast<const uint4*>(row + at);
    } else {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = 0;
#pragma unroll
        for (int j = 0; j < PER_WORD; ++j) {
          const int t = at + i * PER_WORD + j;
          w[i] |= bits_of(t >= 0 && t < V ? row[t] : from_f<T>(-INFINITY)) << (16 * j);
        }
      }
      x.v[k] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}
// (returns whether the CTA has seen a NaN or +inf)
template <typename T>
__device__ __forceinline__ bool scan_stretch(const T* row, int chunk, int V, bool greedy, float c,
                                             const Stored<T>& x, StretchParts& parts) {
  constexpr int VEC = Stored<T>::VEC;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  float top = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int k = 0; k < kScanValues; ++k) {
    top = fmaxf(top, x.at(k));
    bad |= !(x.at(k) < INFINITY);
  }
  top = warp_max(top);
  unsigned long long total = 0;
  int first = V;
  if (greedy) {
    const int t0 = chunk * kScanTokens - static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
#pragma unroll
    for (int k = kScanValues - 1; k >= 0; --k) {
      const int at = t0 + ((k / VEC) * kScanThreads + tid) * VEC + k % VEC;
      if (x.at(k) == top && at >= 0 && at < V) first = at;
    }
    first = __reduce_min_sync(0xffffffffu, first);
  } else {
    const float ref = top == -INFINITY ? 0.f : top;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kScanValues; ++k) sum[k & 3] += ex2((x.at(k) - ref) * c);
    // (bad rows have any sum)
    total = warp_sum_u50(static_cast<unsigned long long>(fminf((sum[0] + sum[1]) + (sum[2] + sum[3]), 64.f) * kSumScale));
  }
  if (lane == 0) parts.top[warp] = top, parts.sum[warp] = total, parts.first[warp] = first;
  return __syncthreads_or(bad) != 0;
}
__device__ __forceinline__ VerifyChunk joined_stretch(const StretchParts& parts, bool bad, float c, int V) {  // warp 0
  const int lane = threadIdx.x & 31;
  const bool in = lane < kScanThreads / 32;
  VerifyChunk out;
  const float top = in ? parts.top[lane] : -INFINITY;
  out.top = warp_max(top);
  unsigned long long total = 0;
  if (in && top > -INFINITY)
    total = static_cast<unsigned long long>(static_cast<float>(parts.sum[lane]) * ex2((top - out.top) * c));
  out.sum = static_cast<long long>(warp_sum_u50(total));
  out.first = __reduce_min_sync(0xffffffffu, in && top == out.top ? parts.first[lane] : V);
  if (bad) out.first = -1;
  return out;
}

// All rows at once.  Where the CTAs run in one round a row's logits are fetched before it is known
// whether they decide anything: 0.6 us less, and the bytes of rows left out cost none.
template <typename T>
__global__ void __launch_bounds__(kScanThreads, kScanPerSm<T>)
    verify_scan_kernel(const __grid_constant__ VerifyArgs a, bool at_once) {
  __shared__ StretchParts parts;
  pdl_trigger();
  pdl_wait();
  const unsigned item = blockIdx.x / static_cast<unsigned>(a.chunks);
  const int chunk = static_cast<int>(blockIdx.x - item * a.chunks);
  const int s = static_cast<int>(item / static_cast<unsigned>(a.rows));
  const int r = static_cast<int>(item - s * static_cast<unsigned>(a.rows));
  if (r == 0 && chunk == 0 && threadIdx.x == 0) a.state[s].done = 0;
  const T* row = row_of<T>(a, s, r);
  Stored<T> x;
  if (at_once) load_stretch(row, chunk, a.V, x);
  const Temperature t = temperature_of(a, s);
  const bool is_draft = r > a.n;
  if (t.bad || (t.greedy && is_draft)) return;  // rows that decide nothing
  const int j = is_draft ? r - a.n - 1 : r;
  if (j > 0 || is_draft) {
    const int have = drafts_of(a, s);
    if (j > have || (is_draft && j == have)) return;
  }
  const float c = log2e_over(t.t);
  if (!at_once) load_stretch(row, chunk, a.V, x);
  const bool bad = scan_stretch(row, chunk, a.V, t.greedy, c, x, parts);
  if (threadIdx.x >= 32) return;
  const VerifyChunk out = joined_stretch(parts, bad, c, a.V);
  if (threadIdx.x == 0) a.stat[(static_cast<size_t>(s) * a.rows + r) * a.chunks + chunk] = out;
}

// Draft by draft over all sequences: a CTA takes one stretch of draft j's rows, the target's and the
// draft's.  Warp 0 of the CTA that ends draft j decides it; what does not stand lowers the
// sequence's stop.  A row is left out only where the stop lies before it, so the rows up to the
// first draft that does not stand are all scanned, whatever the order in which CTAs run.  64 sequences
// of 5 drafts, of which 2.1 stand: 214 of the 361 MB in 52 us.  A CTA's chain bounds it (state, rows,
// sums, count: 5 us with loads on their way for two of them), three CTAs to an SM in float32; one that
// finds its row not wanted takes 1 us.
template <typename T>
__global__ void __launch_bounds__(kScanThreads, kTurnPerSm<T>)
    verify_scan_in_turn_kernel(const __grid_constant__ VerifyArgs a) {
  __shared__ float table[64];
  __shared__ StretchParts parts[2];
  __shared__ int4 s_state;
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31;
  const unsigned level = static_cast<unsigned>(a.S) * a.chunks;
  const int j = static_cast<int>(blockIdx.x / level);
  const unsigned at = blockIdx.x - j * level;
  const int s = static_cast<int>(at / a.chunks), chunk = static_cast<int>(at - s * a.chunks);
  pdl_wait();
  VerifyState* state = after_wait(a.state) + s;
  if (tid == 0) s_state = __ldcg(reinterpret_cast<const int4*>(state));  // (one thread looks: the stop may fall meanwhile)
  __syncthreads();
  const int4 v = s_state;
  if (v.x < j) return;
  const int n = v.y;
  const bool soft = v.z != 0, two = soft && a.draft != nullptr && j < n;
  const float temperature = __int_as_float(v.w), c = log2e_over(temperature);
  const T *row = row_of<T>(a, s, j), *draft_row = two ? row_of<T>(a, s, a.n + 1 + j) : row;
  Stored<T> x, y;
  load_stretch(row, chunk, a.V, x);
  if (two) load_stretch(draft_row, chunk, a.V, y);
  if (tid < 64) table[tid] = kPowers.v[tid];
  const bool bad = scan_stretch(row, chunk, a.V, !soft, c, x, parts[0]);
  const bool draft_bad = two && scan_stretch(draft_row, chunk, a.V, false, c, y, parts[1]);
  if (tid >= 32) return;
  VerifyChunk* stat = a.stat + static_cast<size_t>(s) * a.rows * a.chunks;
  VerifyChunk* p_stat = stat + static_cast<size_t>(j) * a.chunks;
  VerifyChunk* d_stat = stat + static_cast<size_t>(a.n + 1 + j) * a.chunks;
  const VerifyChunk p_out = joined_stretch(parts[0], bad, c, a.V);
  VerifyChunk d_out{};
  if (two) d_out = joined_stretch(parts[1], draft_bad, c, a.V);
  int last = 0;
  if (lane == 0) {
    p_stat[chunk] = p_out;
    if (two) d_stat[chunk] = d_out;
    last = add_acq_rel(&state->scanned[j], 1u) == static_cast<unsigned>(a.chunks) - 1;
  }
  __syncwarp();
  if (__shfl_sync(0xffffffffu, last, 0) == 0) return;
  // this stretch was draft j's last
  const Sequence q = sequence_with(a, Temperature{temperature, !soft, false}, n);
  VerifyRow p, d{0.f, 0.f, 0.f, 0, 0};
  int draft = 0;
  float u = 0.f, xp = 0.f, xq = 0.f;
  if (j < n) {
    draft = after_wait(a.drafts)[static_cast<size_t>(s) * a.n + j];
    u = number_at(a, s, j);
    xp = to_f<T>(row[draft]);
    if (two) xq = to_f<T>(draft_row[draft]);
  }
  if (two && a.chunks <= 16) {  // (the warp's halves take a row each)
    const VerifyChunk* from_stat = lane < 16 ? p_stat : d_stat;
    const VerifyChunk chunk_here = load_chunk(from_stat + min(lane & 15, a.chunks - 1));
    const VerifyRow mine = row_total(from_stat, chunk_here, a.chunks, 16, q, a.V, table);
    auto from = [&](int at) {
      return VerifyRow{__shfl_sync(0xffffffffu, mine.sum_h, at), __shfl_sync(0xffffffffu, mine.sum_l, at),
                       __shfl_sync(0xffffffffu, mine.m, at), __shfl_sync(0xffffffffu, mine.first, at),
                       __shfl_sync(0xffffffffu, mine.ok, at)};
    };
    p = from(0);
    d = from(16);
  } else {
    const int i = min(lane, a.chunks - 1);
    p = row_total(p_stat, load_chunk(p_stat + i), a.chunks, 32, q, a.V, table);
    if (two) d = row_total(d_stat, load_chunk(d_stat + i), a.chunks, 32, q, a.V, table);
  }
  const int what = verdict(q, j, draft, u, xp, xq, p, d, table);
  if (lane == 0) {
    state->target[j] = p;
    state->draft[j] = d;
    state->why[j] = what;
    if (what != kStands) atomicMin(&state->stop, j);
  }
}

__global__ void verify_start_kernel(const __grid_constant__ VerifyArgs a) {
  pdl_trigger();
  pdl_wait();
  const int s = static_cast<int>(blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5));
  if (s >= a.S) return;
  const Temperature t = temperature_of(a, s);
  const int n = drafts_of(a, s), lane = threadIdx.x & 31;
  VerifyState* state = a.state + s;
  if (lane <= kVerifyMaxDrafts) state->scanned[lane] = 0;
  if (lane != 0) return;
  state->stop = t.bad ? -1 : n;
  state->n = n;
  state->soft = !t.greedy;
  state->temperature = t.t;
  state->done = 0;
}

// ---------------------------------------------------------------- the token

constexpr int kFinishWarps = kVerifyWarps, kFinishThreads = 32 * kFinishWarps, kFinishPerSm = 4;
constexpr int kWarpStep = 128, kGroupStep = kFinishWarps * kWarpStep;  // a group, the tokens of a CTA, is a multiple of it
constexpr int kGroupsMost = 128;                                       // groups of a sequence, at most

enum { kFromTarget = 0, kWithout = 1, kResidual = 2 };  // r = p; p without token x; max(p - q, 0)

// floor(u total), u in [0, 1)
__device__ __forceinline__ long long goal_of(float u, long long total) {
  int e;
  const float m = frexpf(u, &e);  // u = m 2^e, m 2^24 a whole number
  const unsigned __int128 v = static_cast<unsigned __int128>(static_cast<uint64_t>(total)) * static_cast<uint32_t>(m * 0x1p24f);
  return 24 - e > 127 ? 0 : static_cast<long long>(v >> (24 - e));
}

__device__ __forceinline__ long long running_sum(long long v) {  // over the warp's lanes, own one included
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += x;
  }
  return v;
}

// A token's share of the sum that the next one is drawn by.
template <typename T>
struct Share {
  const T *p, *q;
  MassRow mp, mq;
  Pair ratio;
  float k, unit;
  int kind, refused;
  const float* table;
  __device__ __forceinline__ long long operator()(long long i, float& x) const {
    x = to_f<T>(p[i]);
    const Pair e = mass(x, mp, table);
    if (kind != kResidual) return i == refused ? 0ll : fixed(e, unit);
    const Pair other = mass(to_f<T>(q[i]), mq, table);
    Pair d = sub(e, mul(other, ratio));
    d.l -= k * other.h;
    return max(fixed(d, unit), 0ll);
  }
};
struct ShareSums {
  long long part[kFinishWarps];
  int first[kFinishWarps], some[kFinishWarps];
};
struct Chosen {
  int token;  // in the thread that has it, else -1
  float x;    // its logit
};

// The CTA's first of `count` tokens from `lo` on whose running sum, that begins with `before`, exceeds
// goal(their whole sum), or where none does the last one with any; a thread keeps KEPT of them.
// `nothing` where the goal is below 0.
template <int KEPT, typename T, typename Goal>
__device__ __forceinline__ Chosen choose(const Share<T>& share, long long lo, int count, long long before, ShareSums& sums,
                                         bool& nothing, Goal&& goal_from) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (count + kFinishThreads - 1) / kFinishThreads, t0 = min(tid * per, count), t1 = min(t0 + per, count);
  long long kept[KEPT > 0 ? KEPT : 1], mine = 0;
  float kept_x[KEPT > 0 ? KEPT : 1], x = 0.f;
#pragma unroll
  for (int i = 0; i < KEPT; ++i) {
    kept[i] = 0;
    if (t0 + i < t1) kept[i] = share(lo + t0 + i, kept_x[i]);
    mine += kept[i];
  }
  for (int i = t0 + KEPT; i < t1; ++i) mine += share(lo + i, x);
  const long long run = running_sum(mine);
  if (lane == 31) sums.part[warp] = run;
  __syncthreads();
  long long base = before, total = 0;
#pragma unroll
  for (int w = 0; w < kFinishWarps; ++w) {
    if (w < warp) base += sums.part[w];
    total += sums.part[w];
  }
  const long long goal = goal_from(total);
  nothing = goal < 0;
  if (nothing) return Chosen{-1, 0.f};
  const unsigned some = __ballot_sync(0xffffffffu, mine > 0);
  const unsigned above = __ballot_sync(0xffffffffu, mine > 0 && base + run > goal);
  if (lane == 0) {
    sums.first[warp] = above != 0 ? tid + __ffs(above) - 1 : -1;
    sums.some[warp] = some != 0 ? tid + 31 - __clz(some) : -1;
  }
  __syncthreads();
  int last = 0, who = -1;
#pragma unroll
  for (int w = kFinishWarps - 1; w >= 0; --w) {
    if (sums.first[w] >= 0) who = sums.first[w];
  }
#pragma unroll
  for (int w = 0; w < kFinishWarps; ++w) {
    if (sums.some[w] >= 0) last = sums.some[w];
  }
  Chosen out{-1, 0.f};
  if (tid != (who >= 0 ? who : last)) return out;
  before = base + run - mine;
  bool found = false;
  auto look = [&](int i, long long v, float x) {
    if (found || v <= 0) return;
    out = Chosen{static_cast<int>(lo + i), x};
    before += v;
    found = before > goal;
  };
#pragma unroll
  for (int i = 0; i < KEPT; ++i) look(t0 + i, kept[i], kept_x[i]);
  for (int i = t0 + KEPT; i < t1 && !found; ++i) {
    const long long v = share(lo + i, x);
    look(i, v, x);
  }
  // (tokens whose sum is more than 0 only by rounding: the last one that the target can give)
  for (long long i = lo + count - 1; out.token < 0; --i) {
    x = to_f<T>(share.p[i]);
    if (i == lo || mass(x, share.mp, share.table).h > 0.f) out = Chosen{static_cast<int>(i), x};
  }
  return out;
}

// All tokens by one CTA, with the exact quotient; from p itself where no more than `least` is left of p - q.
template <typename T>
__device__ __forceinline__ Chosen choose_alone(Share<T> share, int V, float u, float least, ShareSums* sums) {
  bool nothing = true;
  Chosen out{-1, 0.f};
  if (share.kind == kResidual) {
    out = choose<0>(share, 0, V, 0, *sums, nothing,
                    [&](long long total) { return __ll2float_rn(total) > share.unit * least ? goal_of(u, total) : -1ll; });
    __syncthreads();
  }
  if (nothing) {
    share.kind = kFromTarget;
    share.refused = -1;
    out = choose<0>(share, 0, V, 0, *sums, nothing, [&](long long total) { return goal_of(u, total); });
  }
  return out;
}

// Which drafts stand is known in the calls that scan in turn, else worked out here by every CTA
// (2 us).  Packed arithmetic takes two tokens at once; the FMA pipe's share of a token and its draft
// row's is 78 operations.
template <typename T, bool DECIDED>
__global__ void __launch_bounds__(kFinishThreads, kFinishPerSm)
    verify_finish_kernel(const __grid_constant__ VerifyArgs a, int ctas, int group, float unit) {
  __shared__ float table[64];
  __shared__ VerifyRow target[kVerifyMaxDrafts + 1], draft_rows[kVerifyMaxDrafts + 1];
  __shared__ int s_stop, s_why, s_last;
  __shared__ ShareSums s_share;
  __shared__ long long s_part[2][kFinishWarps];
  __shared__ float s_b[kFinishWarps];
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int s = static_cast<int>(blockIdx.x) / ctas, cta = static_cast<int>(blockIdx.x) - s * ctas;
  if (tid < 64) table[tid] = kPowers.v[tid];
  __syncthreads();
  pdl_wait();
  VerifyState* state = after_wait(a.state) + s;
  const float u = number_at(a, s, a.n);
  // (loads that need no other's result first)
  const VerifyChunk* stat = after_wait(a.stat) + static_cast<size_t>(s) * a.rows * a.chunks;
  const int lanes = a.chunks <= 16 ? 16 : 32, per_warp = 32 / lanes;
  auto chunk_of = [&](int r0) {
    const int r = min(r0 + lane / lanes, a.rows - 1);
    return load_chunk(stat + static_cast<size_t>(r) * a.chunks + min(lane & (lanes - 1), a.chunks - 1));
  };
  VerifyChunk chunk{};
  if (!DECIDED) chunk = chunk_of(warp * per_warp);
  Temperature t;
  int n, stop, why;
  if constexpr (DECIDED) {
    const int4 v = *reinterpret_cast<const int4*>(state);
    if (tid <= a.n) target[tid] = state->target[tid], draft_rows[tid] = state->draft[tid];  // (rows left out: anything)
    t = Temperature{__int_as_float(v.w), v.z == 0, v.x < 0};
    n = v.y;
    stop = max(v.x, 0);
    why = t.bad ? kNoTarget : state->why[stop];
  } else {
    t = temperature_of(a, s);
    n = drafts_of(a, s);
  }
  const Sequence q = sequence_with(a, t, n);
  int my_draft = -1;
  if (tid < q.n) my_draft = after_wait(a.drafts)[static_cast<size_t>(s) * a.n + tid];
  if constexpr (DECIDED) {
    __syncthreads();
  } else {
    float my_u = 0.f, xp = 0.f, xq = 0.f;
    if (tid < q.n) {
      my_u = number_at(a, s, tid);
      xp = logit_at<T>(a, s, tid, my_draft);
      if (!q.lookup && q.soft) xq = logit_at<T>(a, s, a.n + 1 + tid, my_draft);
    }
    for (int r0 = warp * per_warp; r0 < a.rows; r0 += kFinishWarps * per_warp) {
      const int r = min(r0 + lane / lanes, a.rows - 1);
      const VerifyRow row = row_total(stat + static_cast<size_t>(r) * a.chunks, chunk, a.chunks, lanes, q, a.V, table);
      if ((lane & (lanes - 1)) == 0) (r <= a.n ? target[r] : draft_rows[r - a.n - 1]) = row;
      if (r0 + kFinishWarps * per_warp < a.rows) chunk = chunk_of(r0 + kFinishWarps * per_warp);
    }
    __syncthreads();
    if (warp == 0) {  // (lane j: draft j)
      const int j = min(lane, a.n);
      int what = verdict(q, j, my_draft, my_u, xp, xq, target[j], draft_rows[j], table);
      const int first = __ffs(__ballot_sync(0xffffffffu, what != kStands || lane >= a.n)) - 1;
      what = __shfl_sync(0xffffffffu, what, first);
      if (lane == 0) s_stop = first, s_why = what;
    }
    __syncthreads();
    stop = s_stop;
    why = s_why;
  }
  // log p of a token with the logit x: (x - m) / t - log(sum), the rounding errors of each kept:
  // log(sum) = g + log(sum exp(-g)) with g near it, and the latter is its argument less 1
  auto log_sum = [&](const VerifyRow& row) {
    const float g = logf(row.sum_h);
    const Pair e = mul(Pair{row.sum_h, row.sum_l}, mass(-g, mass_row(1.f), table));
    return Pair{g, (e.h - 1.f) + e.l};
  };
  auto log_p = [&](float m, const Pair& sum, float x) {
    const float d = x - m, b = d - x, de = (x - (d - b)) + (-m - b);
    const float h = d / q.t.t, l = (fmaf(-h, q.t.t, d) + de) / q.t.t;
    const Pair z = sub(Pair{h, l}, sum);
    return h > -INFINITY ? z.h + z.l : h;
  };
  int32_t* tokens = a.tokens + static_cast<size_t>(s) * (a.n + 1);
  float* logp = a.logp != nullptr ? a.logp + static_cast<size_t>(s) * (a.n + 1) : nullptr;
  if (cta == 0) {
    if (tid <= a.n && tid != stop) {
      tokens[tid] = tid < stop ? my_draft : -1;
      if (logp != nullptr) {
        float lp = 0.f;
        if (tid < stop && q.soft) lp = log_p(target[tid].m, log_sum(target[tid]), logit_at<T>(a, s, tid, my_draft));
        logp[tid] = lp;
      }
    }
    if (tid == 0) {
      a.accepted[s] = stop;
      if (a.lens_out != nullptr) a.lens_out[s] = max(max(after_wait(a.lens)[s], 0) - (a.n - stop), 0);
      if (why == kNoTarget || q.t.greedy) {
        tokens[stop] = why == kNoTarget ? -1 : target[stop].first;
        if (logp != nullptr) logp[stop] = 0.f;
      }
    }
  }
  if (why == kNoTarget || q.t.greedy) return;  // (the same for all CTAs of the sequence)

  const int kind = why == kNoDraft ? kFromTarget : q.lookup ? kWithout : kResidual;
  const VerifyRow row = target[stop], other = draft_rows[stop];
  const T* row_p = row_of<T>(a, s, stop);
  const T* row_q = kind == kResidual ? row_of<T>(a, s, a.n + 1 + stop) : row_p;
  const int refused = kind == kFromTarget ? -1 : after_wait(a.drafts)[static_cast<size_t>(s) * a.n + stop];
  const MassRow mp = row_at(q.factor, row.m), mq = row_at(q.factor, other.m);
  const Pair ratio = kind == kResidual ? div(Pair{row.sum_h, row.sum_l}, Pair{other.sum_h, other.sum_l}) : Pair{0.f, 0.f};

  // this CTA's group of tokens
  VerifyGroup* sums = a.groups + static_cast<size_t>(s) * ctas;
  {
    // (a warp has neighbouring tokens, a lane every 32nd of them)
    const int share = group / kFinishWarps;
    const long long g0 = static_cast<long long>(cta) * group + static_cast<long long>(warp) * share + lane;
    const int left = static_cast<int>(min(static_cast<long long>(share), a.V - g0));  // (from this lane's first token on)
    const Factor2 f2 = factor2(q.factor);
    const uint64_t m2 = both(row.m);
    // Sums of terms above 0, and of those below: each begins at twice the largest that a term can be
    // (E <= 1), so that what a sum's rounding takes off needs no comparison.
    const float most = kind == kResidual ? exp2f(static_cast<float>(max(ilogbf(ratio.h), 0) + 2)) : 2.f;
    Pair2 plus{both(2.f), 0}, minus{both(-most), 0};
    float b = 0.f;
    auto load = [&](const T* from, int i0, float (&x)[4]) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = i0 + k * 32;
        x[k] = i < left ? to_f<T>(from[g0 + i]) : -INFINITY;
      }
    };
    if (kind == kResidual) {
      const uint64_t mq2 = both(other.m), ch = both(ratio.h), nch = both(-ratio.h), cl = both(ratio.l);
      for (int i0 = 0; i0 < share; i0 += kWarpStep) {
        float x[4], y[4];
        load(row_p, i0, x);
        load(row_q, i0, y);
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
          const Pair2 e = mass2(y[k], y[k + 1], mq2, f2, table);
          const Pair2 d = less2(mass2(x[k], x[k + 1], m2, f2, table), e, ch, nch, cl);
          float s0, s1, h0, h1, l0, l1, q0, q1;
          f2unpack(fadd2(d.h, d.l), s0, s1);
          f2unpack(d.h, h0, h1);
          f2unpack(d.l, l0, l1);
          f2unpack(e.h, q0, q1);
          const bool up0 = s0 > 0.f, up1 = s1 > 0.f;
          add_below2(plus, f2pack(up0 ? h0 : 0.f, up1 ? h1 : 0.f), f2pack(up0 ? l0 : 0.f, up1 ? l1 : 0.f));
          add_below2(minus, f2pack(up0 ? 0.f : h0, up1 ? 0.f : h1), f2pack(up0 ? 0.f : l0, up1 ? 0.f : l1));
          b += (up0 ? q0 : 0.f) + (up1 ? q1 : 0.f);
        }
      }
    } else {
      const long long skip = refused - g0;  // the refused token among this thread's
      for (int i0 = 0; i0 < share; i0 += kWarpStep) {
        float x[4];
        load(row_p, i0, x);
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
          const int i = i0 + k * 32;
          const Pair2 e = mass2(i == skip && refused >= 0 ? -INFINITY : x[k],
                                i + 32 == skip && refused >= 0 ? -INFINITY : x[k + 1], m2, f2, table);
          add_below2(plus, e.h, e.l);
        }
      }
    }
    // the two tokens' sums, in units
    auto joined = [&](const Pair2& v, float begin) {
      float h0, h1, l0, l1;
      f2unpack(fsub2(v.h, both(begin)), h0, h1);
      f2unpack(v.l, l0, l1);
      return warp_sum_ll(fixed(Pair{h0, l0}, unit) + fixed(Pair{h1, l1}, unit));
    };
    const long long sum_a = joined(plus, 2.f), sum_d = kind == kResidual ? sum_a + joined(minus, -most) : 0;
    b = warp_sum(b);
    if (lane == 0) s_part[0][warp] = sum_a, s_part[1][warp] = sum_d, s_b[warp] = b;
  }
  __syncthreads();
  if (warp == 0) {
    const bool in = lane < kFinishWarps;
    const long long part_a = in ? s_part[0][lane] : 0;
    const float part_b = in ? s_b[lane] : 0.f;
    const long long sum_a = warp_sum_ll(part_a), sum_d = warp_sum_ll(in ? s_part[1][lane] : 0);
    const float b = warp_sum(part_b);
    VerifyGroup* g = sums + cta;
    if (in) g->warp_a[lane] = part_a, g->warp_b[lane] = part_b;
    if (lane == 0) g->a = sum_a, g->d = sum_d, g->b = b;
    __syncwarp();
    if (lane == 0) s_last = add_acq_rel(&state->done, 1u) == static_cast<unsigned>(ctas) - 1;
  }
  __syncthreads();
  if (!s_last) return;

  // The last CTA: k, the running sums of the groups (each warp for itself, neighbouring groups to
  // a lane), the group that holds the number, the warp's share of it that does, its token.  The
  // place looked for is the first whose running sum exceeds u times the whole.  Groups, shares and
  // tokens are rounded apart: where none does, it is the last one with any.
  constexpr int EACH = kGroupsMost / 32;
  long long group_a[EACH], sd = 0, mine = 0;
  float group_b[EACH];
  const int each = (ctas + 31) / 32, first_g = lane * each;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    group_a[i] = 0;
    group_b[i] = 0.f;
    if (i < each && first_g + i < ctas) {
      const VerifyGroup* g = sums + first_g + i;
      const longlong2 x = __ldcg(reinterpret_cast<const longlong2*>(g));
      group_a[i] = x.x;
      sd += x.y;
      group_b[i] = __ldcg(&g->b);
    }
  }
  const Pair row_log = log_sum(row);  // (while the groups are on their way)
  const float k = kind == kResidual ? __ll2float_rn(warp_sum_ll(sd)) / (unit * other.sum_h) : 0.f;
  auto corrected = [&](long long part, float b) { return max(part - __float2ll_rn(k * b * unit), 0ll); };
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    group_a[i] = corrected(group_a[i], group_b[i]);
    mine += group_a[i];
  }
  long long run = running_sum(mine);
  const long long whole = __shfl_sync(0xffffffffu, run, 31);
  Share<T> share{row_p, row_q, mp, mq, ratio, k, unit, kind, refused, table};
  // What is left of p - q is told from nothing down to `least`: a token's D_i is off by 2^-35.7 of
  // E_p,i + c0 E_q,i at most, all of them by 2^-34.7 of Z_p, and so is the k B that is taken off.
  // At or below it the token is drawn from p.  And where all that is left is not far above k Z_q, tokens
  // whose D_i has another sign than the exact one may be a part of it that counts (rows that
  // are equal but for a few tokens).  Then this CTA goes through all tokens by itself with the exact
  // quotient, 320 us over 128256 of them where rows apart take 18; a draft that was drawn from the
  // draft row is refused over such rows, with 2^13 times k Z_q, once in thousands of calls.
  const float least = row.sum_h * 0x1p-33f;
  const bool alone = kind == kResidual ? __ll2float_rn(whole) <= unit * (least + 0x1p13f * fabsf(k) * other.sum_h) : whole == 0;
  Chosen next;
  if (alone) {
    next = choose_alone(share, a.V, u, least, &s_share);
  } else {
    const long long goal = goal_of(u, whole);
    // the lane of the place looked for, among lanes with running sums `sum` that end with `part` of their own
    auto lane_of = [&](long long part, long long sum) {
      const unsigned some = __ballot_sync(0xffffffffu, part > 0), above = __ballot_sync(0xffffffffu, part > 0 && sum > goal);
      return above != 0 ? __ffs(above) - 1 : 31 - __clz(some);
    };
    int who = lane_of(mine, run), at = 0;
    long long before = run - mine, at_before = before;
    bool found = false;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if (found || group_a[i] == 0) continue;
      at = first_g + i;
      at_before = before;
      before += group_a[i];
      found = before > goal;
    }
    at = __shfl_sync(0xffffffffu, at, who);
    before = __shfl_sync(0xffffffffu, at_before, who);
    long long lo = static_cast<long long>(at) * group;
    const VerifyGroup* g = sums + at;
    const long long part = lane < kFinishWarps ? corrected(__ldcg(&g->warp_a[lane]), __ldcg(&g->warp_b[lane])) : 0;
    run = before + running_sum(part);
    who = max(lane_of(part, run), 0);
    before = __shfl_sync(0xffffffffu, run - part, who);
    const int length = group / kFinishWarps;
    lo += static_cast<long long>(who) * length;
    const int count = static_cast<int>(max(min(static_cast<long long>(length), a.V - lo), 1ll));
    bool nothing;
    next = choose<4>(share, lo, count, before, s_share, nothing, [&](long long) { return goal; });
  }
  if (next.token >= 0) {
    tokens[stop] = next.token;
    if (logp != nullptr) logp[stop] = log_p(row.m, row_log, next.x);
  }
}

// CTAs of a sequence and tokens of a CTA: the shortest groups that come to no more than `rounds`
// rounds of the CTAs that run at once.
struct VerifySlices {
  int ctas, group;
};
VerifySlices verify_slices(int S, int V, int sms, int rounds) {
  const long long at_most = static_cast<long long>(rounds) * kFinishPerSm * sms, all = (V + kGroupStep - 1) / kGroupStep;
  const long long steps = std::min(all, std::max((all + kGroupsMost - 1) / kGroupsMost, (S * all + at_most - 1) / at_most));
  return VerifySlices{static_cast<int>((all + steps - 1) / steps), static_cast<int>(steps) * kGroupStep};
}

// Whether rows are scanned in turn: from 20 stretches to an SM on (128256 float32 logits, drafts of
// which three of five stand, us for all rows and in turn: 8 sequences of 5 drafts 23 and 30, 16 34 and
// 36, 24 49 and 46, 48 82 and 76; 64 of one draft 61 and 56; 16 of 15 drafts 66 and 51).  By the same
// rule: bf16, 24 of 5 drafts 41 and 40, 64 89 and 75; looked-up drafts, 48 of 5 49 and 35; 32003 logits, 64
// of 5 (18 to an SM) 33 and 36, 100 48 and 47; 1000 logits, 700 of 5 55 and 53.  It does not pay for
// one draft over rows shorter than a stretch: 1100 sequences of 1000 logits 38 and 45, 1700 of 50
// with drafts looked up 44 and 52.
bool in_turn(const VerifyArgs& a, int sms) {
  return a.n > 0 && static_cast<long long>(a.S) * a.rows * a.chunks > 20ll * sms;
}

template <typename T>
cudaError_t run_verify(const VerifyArgs& a, int sms, cudaStream_t s) {
  // Two rounds where the decisions have been made: CTAs of sequences that end at once make room
  // (64 sequences, us: one round 90, two 81, three 82); one where every CTA makes them (24
  // sequences of 50257 bf16 logits: one 19.9, two 23.5, with logits unpacked).
  const bool turns = in_turn(a, sms);
  const VerifySlices c = verify_slices(a.S, a.V, sms, turns ? 2 : 1);
  int bits = 10;  // units in which sums of up to V exponentials stay below 2^62
  while ((1 << bits) < a.V) ++bits;
  const float unit = std::ldexp(1.f, 62 - bits);
  const dim3 grid(static_cast<unsigned>(a.S) * a.rows * a.chunks), finish(static_cast<unsigned>(a.S) * c.ctas);
  if (turns) {
    ZSAA_LAUNCH(verify_start_kernel, dim3((a.S + 7) / 8), dim3(256), 0, s, a);
    const dim3 turns_grid(static_cast<unsigned>(a.S) * (a.n + 1) * a.chunks);
    ZSAA_LAUNCH(verify_scan_in_turn_kernel<T>, turns_grid, dim3(kScanThreads), 0, s, a);
    ZSAA_LAUNCH((verify_finish_kernel<T, true>), finish, dim3(kFinishThreads), 0, s, a, c.ctas, c.group, unit);
  } else {
    ZSAA_LAUNCH(verify_scan_kernel<T>, grid, dim3(kScanThreads), 0, s, a, grid.x <= static_cast<unsigned>(kScanPerSm<T> * sms));
    ZSAA_LAUNCH((verify_finish_kernel<T, false>), finish, dim3(kFinishThreads), 0, s, a, c.ctas, c.group, unit);
  }
  return cudaSuccess;
}

}  // namespace

// one more than the tokens fill: a row may start inside a 16-byte block
int verify_chunks(int V) { return (V + 7 + kScanTokens - 1) / kScanTokens; }
int verify_groups_most(int V) { return std::min((V + kGroupStep - 1) / kGroupStep, kGroupsMost); }

cudaError_t launch_draft_verify(const VerifyArgs& a, int dtype, int sms, cudaStream_t s) {
  return dtype == ZSAA_F32 ? run_verify<float>(a, sms, s) : run_verify<bf16>(a, sms, s);
}

}  // namespace zsaa
