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
//   verify_sample_kernel  one cluster per sequence: which drafts stand, then the token.
//
// What decides a draft is one comparison of two quotients, off by about 1e-8 with sums of
// float32 exponentials.  What decides a token is where u_n falls among V borders, some 1e-5
// apart and closer: a running sum that is off by 1e-9 picks the wrong token every few thousand
// calls.  So the rows at which a sequence stops are gone through again with exponentials as
// pairs of floats, good to about 2^-37, and sums in pairs and in 64 bits.
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

template <typename T>
__global__ void __launch_bounds__(kScanThreads, 4) verify_scan_kernel(const __grid_constant__ VerifyArgs a, int rows) {
  constexpr int VEC = 16 / sizeof(T), VECS = kScanValues / VEC;
  __shared__ float s_top[kScanThreads / 32];
  __shared__ double s_sum[kScanThreads / 32];
  __shared__ int s_first[kScanThreads / 32];
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const unsigned item = blockIdx.x / static_cast<unsigned>(a.chunks);
  const int chunk = static_cast<int>(blockIdx.x - item * a.chunks);
  const int s = static_cast<int>(item / static_cast<unsigned>(rows)), r = static_cast<int>(item - s * static_cast<unsigned>(rows));
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
  if (lane == 0) s_top[warp] = top;
  bad = __syncthreads_or(bad) != 0;
#pragma unroll
  for (int w = 0; w < kScanThreads / 32; ++w) top = fmaxf(top, s_top[w]);
  double total = 0.0;
  int first = a.V;
  if (t.greedy) {
#pragma unroll
    for (int k = kScanValues - 1; k >= 0; --k) {
      const int at = t0 + ((k / VEC) * kScanThreads + tid) * VEC + k % VEC;
      if (x[k] == top && at >= 0 && at < a.V) first = at;
    }
    first = __reduce_min_sync(0xffffffffu, first);
  } else {
    const float c = static_cast<float>(1.4426950408889634 / static_cast<double>(t.t));
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < kScanValues; ++k) sum += ex2((x[k] - ref) * c);
    total = sum;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  }
  if (lane == 0) s_sum[warp] = total, s_first[warp] = first;
  __syncthreads();
  if (tid == 0) {
    VerifyChunk out{};
#pragma unroll
    for (int w = 0; w < kScanThreads / 32; ++w) {
      out.sum += s_sum[w];
      first = min(first, s_first[w]);
    }
    out.top = top;
    out.first = first;
    out.bad = bad;
    a.stat[(static_cast<size_t>(s) * rows + r) * a.chunks + chunk] = out;
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
  const double c = 1.4426950408889634074 / static_cast<double>(t);
  const float ch = static_cast<float>(c);
  return MassRow{m, ch, static_cast<float>(c - static_cast<double>(ch))};
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

// running sums of pairs
__device__ __forceinline__ void add(Pair& s, float h, float l) {
  const float t = s.h + h, b = t - s.h;
  s.l += ((s.h - (t - b)) + (h - b)) + l;
  s.h = t;
}
__device__ __forceinline__ double value(const Pair& s) { return static_cast<double>(s.h) + static_cast<double>(s.l); }

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// ---------------------------------------------------------------- decisions and the token

constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32, kSampleCtas = 8;
constexpr int kGroups = 4;  // a warp's tokens in so many groups, each with its sum
constexpr int kSums = kSampleCtas * kSampleWarps * kGroups;

enum { kFromTarget = 0, kWithout = 1, kResidual = 2 };  // r = p; p without token x; max(p - q, 0)

struct RowStat {
  double sum;
  float top;
  int first;
  int ok;  // the row has a distribution
};

__device__ __forceinline__ void st_cluster_f64(uint32_t saddr, uint32_t rank, double v) {
  asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(map_rank(saddr, rank)), "d"(v) : "memory");
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads, 1) verify_sample_kernel(const __grid_constant__ VerifyArgs a, int rows) {
  __shared__ float table_h[32], table_l[32];
  __shared__ RowStat stat[2 * kVerifyMaxDrafts + 1];
  __shared__ int s_stands[kVerifyMaxDrafts + 1];
  __shared__ double part[2][kSampleWarps];
  __shared__ double norm[2][kSampleCtas];
  __shared__ double sums[2][kSums];
  __shared__ int s_segment;
  __shared__ double s_before;
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctas = static_cast<int>(cluster_size()), rank = static_cast<int>(cluster_rank());
  const int s = static_cast<int>(blockIdx.x) / ctas;
  if (tid < 32) {
    const double e = exp2(tid / 32.0);
    table_h[tid] = static_cast<float>(e);
    table_l[tid] = static_cast<float>(e - static_cast<double>(table_h[tid]));
  }
  cluster_sync_all();  // every CTA of the cluster runs before another writes into it
  pdl_wait();
  const Temperature t = temperature_of(a, s);
  const int n = drafts_of(a, s);
  const bool lookup = a.draft == nullptr;
  const VerifyChunk* chunks = after_wait(a.stat) + static_cast<size_t>(s) * rows * a.chunks;
  const double inv_t = t.greedy || t.bad ? 1.0 : 1.0 / static_cast<double>(t.t);

  // every row that may decide something: its maximum and its sum
  for (int r = warp; r < rows; r += kSampleWarps) {
    const bool is_draft = r > a.n;
    RowStat out{0.0, -INFINITY, a.V, 0};
    if (!t.bad && (is_draft ? !t.greedy && r - a.n - 1 < n : r <= n)) {
      const VerifyChunk* c = chunks + static_cast<size_t>(r) * a.chunks;
      int bad = 0;
      for (int i = lane; i < a.chunks; i += 32) {
        out.top = fmaxf(out.top, c[i].top);
        bad |= c[i].bad;
      }
      out.top = warp_max(out.top);
      double sum = 0.0;
      for (int i = lane; i < a.chunks; i += 32) {
        if (c[i].top == -INFINITY) continue;
        if (t.greedy) {
          if (c[i].top == out.top) out.first = min(out.first, c[i].first);
        } else {
          sum += c[i].sum * exp((static_cast<double>(c[i].top) - static_cast<double>(out.top)) * inv_t);
        }
      }
      out.sum = warp_sum64(sum);
      out.first = __reduce_min_sync(0xffffffffu, out.first);
      out.ok = __reduce_or_sync(0xffffffffu, bad) == 0 && out.top > -INFINITY;
    }
    if (lane == 0) stat[r] = out;
  }
  __syncthreads();
  auto log_p = [&](int r, int x) {  // of token x in row r, natural
    const double d = static_cast<double>(to_f<T>(row_of<T>(a, s, r)[x])) - static_cast<double>(stat[r].top);
    return d * inv_t - log(stat[r].sum);
  };
  const int32_t* drafts = after_wait(a.drafts) + static_cast<size_t>(s) * a.n;
  const float* uniform = after_wait(a.uniform) + static_cast<size_t>(s) * (a.n + 1);
  // numbers outside [0, 1) count as the nearest ones in it, a NaN as 0
  auto number = [&](int j) { return static_cast<double>(fminf(fmaxf(uniform[j], 0.f), 0x1.fffffep-1f)); };
  enum { kStands, kRefused, kNoDraft, kNoTarget };
  if (tid <= a.n) {
    int what = kNoDraft;
    if (!stat[tid].ok && tid <= n) {
      what = kNoTarget;
    } else if (tid < n) {
      const int x = drafts[tid];
      if (t.greedy) {
        what = stat[tid].first == x ? kStands : kRefused;
      } else if (lookup) {
        what = number(tid) < exp(log_p(tid, x)) ? kStands : kRefused;
      } else if (stat[a.n + 1 + tid].ok) {
        const double lq = log_p(a.n + 1 + tid, x), lp = log_p(tid, x);
        // (q(x) = 0: it stands where p(x) > 0)
        what = lp > -INFINITY && (lq == -INFINITY || number(tid) < exp(lp - lq)) ? kStands : kRefused;
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
  if (rank == 0) {
    if (tid <= a.n && tid != stop) {
      tokens[tid] = tid < stop ? drafts[tid] : -1;
      if (logp != nullptr) logp[tid] = tid < stop && !t.greedy ? static_cast<float>(log_p(tid, drafts[tid])) : 0.f;
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
  if (why == kNoTarget || t.greedy) return;  // (the same for the whole cluster)

  const T* row_p = row_of<T>(a, s, stop);
  int kind = why == kNoDraft ? kFromTarget : lookup ? kWithout : kResidual;
  const T* row_q = kind == kResidual ? row_of<T>(a, s, a.n + 1 + stop) : row_p;
  const int refused = kind == kFromTarget ? -1 : drafts[stop];
  const MassRow mp = mass_row(stat[stop].top, t.t);
  const MassRow mq = kind == kResidual ? mass_row(stat[a.n + 1 + stop].top, t.t) : mp;
  // tokens of a warp: kGroups groups of `group`, a multiple of 32
  const int warps = ctas * kSampleWarps, gw = rank * kSampleWarps + warp;
  const int group = ((a.V + warps * kGroups - 1) / (warps * kGroups) + 31) & ~31;
  const long long w0 = static_cast<long long>(gw) * kGroups * group;

  Pair ratio{0.f, 0.f};  // sum_p / sum_q
  if (kind == kResidual) {
    Pair sp{0.f, 0.f}, sq{0.f, 0.f};
#pragma unroll 2
    for (int i = lane; i < kGroups * group; i += 32) {
      if (w0 + i >= a.V) break;
      const Pair p = mass(to_f<T>(row_p[w0 + i]), mp, table_h, table_l), q = mass(to_f<T>(row_q[w0 + i]), mq, table_h, table_l);
      add(sp, p.h, p.l);
      add(sq, q.h, q.l);
    }
    const double p = warp_sum64(value(sp)), q = warp_sum64(value(sq));
    if (lane == 0) part[0][warp] = p, part[1][warp] = q;
    __syncthreads();
    if (tid < 2) {
      double v = 0.0;
      for (int w = 0; w < kSampleWarps; ++w) v += part[tid][w];
      for (int r = 0; r < ctas; ++r) st_cluster_f64(smem_u32(&norm[tid][rank]), r, v);
    }
    cluster_sync_all();
    double np = 0.0, nq = 0.0;
    for (int r = 0; r < ctas; ++r) np += norm[0][r], nq += norm[1][r];
    const double x = np / nq;
    ratio.h = static_cast<float>(x);
    ratio.l = static_cast<float>(x - static_cast<double>(ratio.h));
  }

  // r of a token, times the sum of p's exponentials
  auto left = [&](long long i) {
    const Pair p = mass(to_f<T>(row_p[i]), mp, table_h, table_l);
    if (kind == kFromTarget) return p;
    if (kind == kWithout) return i == refused ? Pair{0.f, 0.f} : p;
    const Pair q = mass(to_f<T>(row_q[i]), mq, table_h, table_l);
    const float qh = __fmul_rn(q.h, ratio.h), ql = fmaf(q.h, ratio.h, -qh) + fmaf(q.h, ratio.l, q.l * ratio.h);
    const float h = p.h - qh, b = h - p.h;
    const float l = ((p.h - (h - b)) + (-qh - b)) + (p.l - ql);
    return h + l > 0.f ? Pair{h, l} : Pair{0.f, 0.f};
  };
  int turn = 0;
  double total = 0.0;
  for (;;) {
    for (int g = 0; g < kGroups; ++g) {
      Pair sum{0.f, 0.f};
      for (int i = lane; i < group; i += 32) {
        const long long at = w0 + static_cast<long long>(g) * group + i;
        if (at >= a.V) break;
        const Pair r = left(at);
        add(sum, r.h, r.l);
      }
      const double v = warp_sum64(value(sum));
      if (lane < ctas) st_cluster_f64(smem_u32(&sums[turn][gw * kGroups + g]), lane, v);
    }
    cluster_sync_all();
    total = 0.0;
    if (warp == 0) {  // running sums, a lane per stretch of them
      const int all = warps * kGroups, each = all / 32;
      double mine = 0.0;
      for (int i = 0; i < each; ++i) mine += sums[turn][lane * each + i];
      double run = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double x = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += x;
      }
      total = __shfl_sync(0xffffffffu, run, 31);
      const double goal = number(a.n) * total;
      const unsigned above = __ballot_sync(0xffffffffu, run > goal);
      const int who = above != 0 ? __ffs(above) - 1 : 31;
      if (lane == who) {
        // (its own sums may round otherwise than the running one: then its last with any)
        double before = run - mine;
        int at = -1;
        double at_before = before;
        for (int i = 0; i < each; ++i) {
          const double v = sums[turn][lane * each + i];
          if (v > 0.0) at = lane * each + i, at_before = before;
          before += v;
          if (before > goal && v > 0.0) break;
        }
        s_segment = at;
        s_before = at_before;
      }
      if (lane == 0) part[0][0] = total;
    }
    __syncthreads();
    total = part[0][0];
    if (total > 0.0 || kind == kFromTarget) break;
    kind = kFromTarget;  // p = q as far as can be told: nothing is left of p - q
    turn = 1;
  }
  // the segment's warp finds the token
  const int segment = s_segment;
  if (segment < 0 || segment / kGroups != gw) return;
  const double goal = number(a.n) * total;
  double before = s_before;
  int token = -1;
  for (int i = lane; i - lane < group; i += 32) {
    const long long at = static_cast<long long>(segment) * group + i;
    double r = 0.0;
    if (at < a.V) r = value(left(at));
    double run = r;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double x = __shfl_up_sync(0xffffffffu, run, o);
      if (lane >= o) run += x;
    }
    const unsigned some = __ballot_sync(0xffffffffu, r > 0.0);
    const unsigned above = __ballot_sync(0xffffffffu, r > 0.0 && before + run > goal);
    if (above != 0) {
      token = static_cast<int>(at - lane) + __ffs(above) - 1;
      break;
    }
    if (some != 0) token = static_cast<int>(at - lane) + 31 - __clz(some);
    before += __shfl_sync(0xffffffffu, run, 31);
  }
  if (lane == 0) {
    tokens[stop] = token;
    if (logp != nullptr) logp[stop] = static_cast<float>(log_p(stop, token));
  }
}

template <typename T>
cudaError_t run_verify(const VerifyArgs& a, cudaStream_t s) {
  const int rows = a.n + 1 + (a.draft != nullptr ? a.n : 0);
  const unsigned grid = static_cast<unsigned>(a.S) * rows * a.chunks;
  ZSAA_LAUNCH(verify_scan_kernel<T>, dim3(grid), dim3(kScanThreads), 0, s, a, rows);
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.S) * kSampleCtas);
  cfg.blockDim = dim3(kSampleThreads);
  cfg.stream = s;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kSampleCtas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, verify_sample_kernel<T>, a, rows);
}

}  // namespace

// one more than the tokens fill: a row may start inside a 16-byte block
int verify_chunks(int V) { return (V + 7 + kScanTokens - 1) / kScanTokens; }

cudaError_t launch_draft_verify(const VerifyArgs& a, int dtype, cudaStream_t s) {
  return dtype == ZSAA_F32 ? run_verify<float>(a, s) : run_verify<bf16>(a, s);
}

}  // namespace zsaa
