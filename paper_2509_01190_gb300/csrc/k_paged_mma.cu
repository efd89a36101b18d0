// Attention over a paged cache on mma.sync: tiles of 16 query rows against the keys of an
// entry; few rows in bf16 (m16n8k16), any number in float32 (m16n8k8).
//
// A decode step has n_q * (Hq / Hkv) rows to each KV head, 4 or 8 as a rule, so the
// keys and values stream past once and the tensor work is small: the kernel is bound
// by HBM on long caches and by its chain of loads on short ones.  Each of the 4 warps
// walks its own 16 keys (float32: 8) of every block with a ring of cp.async stages of its
// own, so nothing but the end of a part synchronises the CTA; a warp's keys never leave a
// page.  The ring runs ahead over the ends of parts: a CTA with several short items has the
// next item's keys in flight while it joins its warps' results of the last.
//
// Per tile of keys: S = Q K^T, the running maximum (moved only when the tile's exceeds it by
// 2^8: P entries up to 256 are exact in float32 and in the pair), P = 2^(S scale - m), and
// O += P V in float32.  In bf16, P is carried as the pair P_hi + P_lo (one bf16 would cost
// 0.1% in every output).
//
// float32 operands are split into pairs of tf32: x = hi + lo, hi the nearest number of 11
// significant bits, lo the rest cut to 11.  The rest has a sign and 12 bits, so at most the last
// bit of x is lost, 2^-23 |x| (a rounding to 11 would lose no less).  A NaN stays one in lo.  The
// products hi hi, hi lo and lo hi are taken and lo lo, at most 2^-22 of the product, is not.  The
// tensor cores' own sums may be rounded towards zero, so no sum of hi hi is longer than four
// of them (32 dims): scores are put together from such sums, and a tile's P V is added to the
// output, in float32 additions.  (The sums of the other two, 2^-11 of those, run over all dims.)
//
// 48 sequences of 2000 to 4000 bf16 entries, 8 heads of 128 dims: 95 us for 576 MB, 90% of the
// copy rate.  float32, 64 sequences of 2048: 216 us for 1.07 GB, 73%; with more rows than 16 to a
// head it is bound by the chain of a warp's tile (96 products for 8 keys at 128 dims), 1 us
// with two warps on an SM's quarter.
#include <algorithm>

#include "paged.cuh"

namespace zsaa {
namespace {

constexpr int MM_WARPS = 4, MM_THREADS = 32 * MM_WARPS, MM_ROWS = 16;
constexpr int MM_STAGES = 3;
constexpr int MM_JOIN = 1024;  // floats of a warp in the buffer that joins results: 8 rows of 128 dims, 16 of 64
constexpr float MM_RESCALE_LOG2 = 8.f;

template <typename T, int HD>
struct MmCfg {
  static constexpr int KEYS = 32 / sizeof(T);    // of a warp's tile
  static constexpr int BLOCK = KEYS * MM_WARPS;  // of a block
  static constexpr int TILE = KEYS * HD * static_cast<int>(sizeof(T));  // bytes of a tile's keys, or their values
  static constexpr int RING = MM_STAGES * 2 * TILE;  // a warp's
  static constexpr int JOIN = MM_WARPS * MM_JOIN * 4;
  static constexpr int SMEM = MM_WARPS * RING + JOIN;
  static constexpr int CTAS = HD == 128 ? 2 : HD == 64 ? 3 : 4;  // resident per SM
};

// byte offset of 16-byte chunk c of row r, chunks XOR-swizzled by the row (conflict-free ldmatrix)
template <int HD>
__device__ __forceinline__ uint32_t mm_swz(int r, int c) {
  return static_cast<uint32_t>(r * HD * 2 + ((c ^ (r & 7)) << 4));
}

// A warp's rows: queries as the A operand (rows gid and gid + 8, dims 2 tig, 2 tig + 1 and
// those + 8 of every 16), accumulators, and maximum and sum of rows gid and gid + 8 (the sum
// of this thread's keys alone).
template <typename T, int HD>
struct MmRows;
template <int HD>
struct MmRows<bf16, HD> {
  uint32_t q[HD / 16][4];
  float o[HD / 8][4];
  float m[2], l[2];
};
// float32: a product's 8 terms are dims 16 j + 4 tig + 2 (t & 1), + 1 of the four tig, for
// t = 2 j or 2 j + 1, so that a thread's dims of a key lie together; o[4 i + k] has dims
// 32 i + 8 tig + k and those + 4
template <int HD>
struct MmRows<float, HD> {
  uint32_t qh[HD / 8][4], ql[HD / 8][4];
  float o[HD / 8][4];
  float m[2], l[2];
};
template <typename T, int HD>
__device__ __forceinline__ void mm_clear(MmRows<T, HD>& x) {
#pragma unroll
  for (int i = 0; i < HD / 8; ++i) x.o[i][0] = x.o[i][1] = x.o[i][2] = x.o[i][3] = 0.f;
  x.m[0] = x.m[1] = -INFINITY;
  x.l[0] = x.l[1] = 0.f;
}
// q0, q1: rows gid and gid + 8; in0, in1: whether there are such
template <int HD>
__device__ __forceinline__ void mm_load_q(MmRows<bf16, HD>& x, const bf16* q0, const bf16* q1, bool in0, bool in1) {
  const int tig = threadIdx.x & 3;
#pragma unroll
  for (int kk = 0; kk < HD / 16; ++kk) {
    x.q[kk][0] = in0 ? *reinterpret_cast<const uint32_t*>(q0 + 16 * kk + 2 * tig) : 0u;
    x.q[kk][1] = in1 ? *reinterpret_cast<const uint32_t*>(q1 + 16 * kk + 2 * tig) : 0u;
    x.q[kk][2] = in0 ? *reinterpret_cast<const uint32_t*>(q0 + 16 * kk + 8 + 2 * tig) : 0u;
    x.q[kk][3] = in1 ? *reinterpret_cast<const uint32_t*>(q1 + 16 * kk + 8 + 2 * tig) : 0u;
  }
}
__device__ __forceinline__ void mm_split(float x, uint32_t& hi, uint32_t& lo) {
  hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;  // (the carry makes a zero of some NaNs)
  lo = __float_as_uint(x - __uint_as_float(hi)) & 0xffffe000u;  // (cut: 0x7fffffff, the NaN of a difference, stays NaN)
}
template <int HD>
__device__ __forceinline__ void mm_load_q(MmRows<float, HD>& x, const float* q0, const float* q1, bool in0, bool in1) {
  const int tig = threadIdx.x & 3;
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int j = 0; j < HD / 16; ++j) {
    const float4 u = in0 ? *reinterpret_cast<const float4*>(q0 + 16 * j + 4 * tig) : zero;
    const float4 v = in1 ? *reinterpret_cast<const float4*>(q1 + 16 * j + 4 * tig) : zero;
    mm_split(u.x, x.qh[2 * j][0], x.ql[2 * j][0]);
    mm_split(v.x, x.qh[2 * j][1], x.ql[2 * j][1]);
    mm_split(u.y, x.qh[2 * j][2], x.ql[2 * j][2]);
    mm_split(v.y, x.qh[2 * j][3], x.ql[2 * j][3]);
    mm_split(u.z, x.qh[2 * j + 1][0], x.ql[2 * j + 1][0]);
    mm_split(v.z, x.qh[2 * j + 1][1], x.ql[2 * j + 1][1]);
    mm_split(u.w, x.qh[2 * j + 1][2], x.ql[2 * j + 1][2]);
    mm_split(v.w, x.qh[2 * j + 1][3], x.ql[2 * j + 1][3]);
  }
}
// A thread's results into rows gid and gid + 8 (where there are such) of a buffer of `dims`
// floats a row, dims d0 on; a row's groups of 8 floats are XORed by its number, which keeps
// stores and loads clear of bank conflicts.
template <int HD>
__device__ __forceinline__ void mm_put(const MmRows<bf16, HD>& x, float* row0, float* row8, int d0, int dims, bool in0, bool in1) {
  const int lane = threadIdx.x & 31, flip = (lane >> 2 & 3) * 8, tig = lane & 3;
#pragma unroll
  for (int i = 0; i < HD / 8; ++i)
    if (8 * i >= d0 && 8 * i < d0 + dims) {
      const int c = ((8 * i - d0) ^ flip) + 2 * tig;
      if (in0) *reinterpret_cast<float2*>(row0 + c) = make_float2(x.o[i][0], x.o[i][1]);
      if (in1) *reinterpret_cast<float2*>(row8 + c) = make_float2(x.o[i][2], x.o[i][3]);
    }
}
template <int HD>
__device__ __forceinline__ void mm_put(const MmRows<float, HD>& x, float* row0, float* row8, int d0, int dims, bool in0, bool in1) {
  const int lane = threadIdx.x & 31, flip = (lane >> 2 & 3) * 8, tig = lane & 3;
#pragma unroll
  for (int i = 0; i < HD / 32; ++i)
    if (32 * i >= d0 && 32 * i < d0 + dims) {
      const int c = (32 * i + 8 * tig - d0) ^ flip;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (in0)
          *reinterpret_cast<float4*>(row0 + c + 4 * k) = make_float4(x.o[4 * i][k], x.o[4 * i + 1][k], x.o[4 * i + 2][k], x.o[4 * i + 3][k]);
        if (in1)
          *reinterpret_cast<float4*>(row8 + c + 4 * k) =
              make_float4(x.o[4 * i][2 + k], x.o[4 * i + 1][2 + k], x.o[4 * i + 2][2 + k], x.o[4 * i + 3][2 + k]);
      }
    }
}
// byte offsets of 16-byte chunk c of a tile's row r: keys and values, free of bank conflicts
// as mm_tile reads them
template <typename T, int HD>
__device__ __forceinline__ uint32_t mm_key(int r, int c) {
  if constexpr (sizeof(T) == 2) return mm_swz<HD>(r, c);
  return static_cast<uint32_t>(r * HD * 4 + ((c ^ (r & 1) << 2) << 4));
}
template <typename T, int HD>
__device__ __forceinline__ uint32_t mm_value(int r, int c) {
  if constexpr (sizeof(T) == 2) return mm_swz<HD>(r, c);
  return static_cast<uint32_t>(r * HD * 4 + ((c ^ (r >> 1 & 3) << 1) << 4));
}
// Asks for a tile's keys and their values, which lie one after the other from element `at`
// on; rows past `keys` are zero.
template <typename T, int HD>
__device__ __forceinline__ void mm_load_tile(const PagedArgs& a, uint32_t sk, size_t at, int keys) {
  using C = MmCfg<T, HD>;
  constexpr int E = 16 / sizeof(T), CH = HD / E, STEP = 32 / CH;  // elements of a chunk, chunks per row, rows per round
  const int lane = threadIdx.x & 31, c = lane % CH;
  const uint32_t sv = sk + C::TILE;
#pragma unroll
  for (int i = 0; i < C::KEYS / STEP; ++i) {
    const int r = lane / CH + i * STEP;
    const size_t from = at + static_cast<size_t>(r < keys ? r : 0) * HD + c * E;
    cp_async16(sk + mm_key<T, HD>(r, c), static_cast<const T*>(a.k) + from, r < keys);
    cp_async16(sv + mm_value<T, HD>(r, c), static_cast<const T*>(a.v) + from, r < keys);
  }
}
// 16 keys (the first `keys` count) and their values at sk
template <int HD>
__device__ __forceinline__ void mm_tile(MmRows<bf16, HD>& x, uint32_t sk, int keys, float scale) {
  const int lane = threadIdx.x & 31, tig = lane & 3, mi = lane >> 3;
  const uint32_t sv = sk + MmCfg<bf16, HD>::TILE;
  float s[2][4] = {};
#pragma unroll
  for (int kk = 0; kk < HD / 16; ++kk) {
    uint32_t b0, b1, b2, b3;
    ldsm_x4(sk + mm_swz<HD>((mi >> 1) * 8 + (lane & 7), kk * 2 + (mi & 1)), b0, b1, b2, b3);
    mma_bf16_16816(s[0], x.q[kk], b0, b1);
    mma_bf16_16816(s[1], x.q[kk], b2, b3);
  }
  float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[t][e] = 8 * t + 2 * tig + (e & 1) < keys ? s[t][e] * scale : -INFINITY;
      mx[e >> 1] = fmaxf(mx[e >> 1], s[t][e]);
    }
  bool need = false;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
    mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
    need |= mx[i] > x.m[i] + MM_RESCALE_LOG2;
  }
  if (__any_sync(0xffffffffu, need)) {
    float f[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float mn = fmaxf(x.m[i], mx[i]);
      f[i] = mn == -INFINITY ? 1.f : ex2_fast(x.m[i] - mn);
      x.m[i] = mn;
      x.l[i] *= f[i];
    }
#pragma unroll
    for (int i = 0; i < HD / 8; ++i) {
      x.o[i][0] *= f[0];
      x.o[i][1] *= f[0];
      x.o[i][2] *= f[1];
      x.o[i][3] *= f[1];
    }
  }
  const float base[2] = {x.m[0] == -INFINITY ? 0.f : x.m[0], x.m[1] == -INFINITY ? 0.f : x.m[1]};
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float p0 = ex2_fast(s[t][2 * i] - base[i]), p1 = ex2_fast(s[t][2 * i + 1] - base[i]);
      x.l[i] += p0 + p1;
      const uint32_t u = pack_bf16x2(p0, p1);
      hi[2 * t + i] = u;
      lo[2 * t + i] = pack_bf16x2(p0 - bf16lo(u), p1 - bf16hi(u));
    }
#pragma unroll
  for (int d = 0; d < HD / 16; ++d) {
    uint32_t b0, b1, b2, b3;
    ldsm_x4_t(sv + mm_swz<HD>((mi & 1) * 8 + (lane & 7), d * 2 + (mi >> 1)), b0, b1, b2, b3);
    mma_bf16_16816(x.o[2 * d], hi, b0, b1);
    mma_bf16_16816(x.o[2 * d + 1], hi, b2, b3);
    mma_bf16_16816(x.o[2 * d], lo, b0, b1);
    mma_bf16_16816(x.o[2 * d + 1], lo, b2, b3);
  }
}

__device__ __forceinline__ void mma_tf32_1688(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mm_lds4(uint32_t at, float (&x)[4]) {
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]) : "r"(at) : "memory");
}
// 8 keys (the first `keys` count) and their values at sk
template <int HD>
__device__ __forceinline__ void mm_tile(MmRows<float, HD>& x, uint32_t sk, int keys, float scale) {
  const int lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  const uint32_t sv = sk + MmCfg<float, HD>::TILE;
  float s[4] = {}, hl[4] = {}, lh[4] = {};
#pragma unroll
  for (int j0 = 0; j0 < HD / 16; j0 += 2) {
    float hh[4] = {};
#pragma unroll
    for (int j = j0; j < j0 + 2; ++j) {
      float y[4];
      uint32_t h[4], l[4];
      mm_lds4(sk + mm_key<float, HD>(gid, 4 * j + tig), y);
#pragma unroll
      for (int e = 0; e < 4; ++e) mm_split(y[e], h[e], l[e]);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        mma_tf32_1688(hh, x.qh[2 * j + t], h[2 * t], h[2 * t + 1]);
        mma_tf32_1688(hl, x.qh[2 * j + t], l[2 * t], l[2 * t + 1]);
        mma_tf32_1688(lh, x.ql[2 * j + t], h[2 * t], h[2 * t + 1]);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] += hh[e];
  }
  float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    s[e] = 2 * tig + (e & 1) < keys ? (s[e] + (hl[e] + lh[e])) * scale : -INFINITY;
    mx[e >> 1] = fmaxf(mx[e >> 1], s[e]);
  }
  bool need = false;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
    mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
    need |= mx[i] > x.m[i] + MM_RESCALE_LOG2;
  }
  if (__any_sync(0xffffffffu, need)) {
    float f[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float mn = fmaxf(x.m[i], mx[i]);
      f[i] = mn == -INFINITY ? 1.f : exp2f(x.m[i] - mn);
      x.m[i] = mn;
      x.l[i] *= f[i];
    }
#pragma unroll
    for (int i = 0; i < HD / 8; ++i) {
      x.o[i][0] *= f[0];
      x.o[i][1] *= f[0];
      x.o[i][2] *= f[1];
      x.o[i][3] *= f[1];
    }
  }
  uint32_t ph[4], pl[4];  // keys 2 tig and 2 tig + 1 as terms tig and tig + 4 of the product
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float base = x.m[i] == -INFINITY ? 0.f : x.m[i];
    const float p0 = exp2f(s[2 * i] - base), p1 = exp2f(s[2 * i + 1] - base);
    x.l[i] += p0 + p1;
    mm_split(p0, ph[i], pl[i]);
    mm_split(p1, ph[2 + i], pl[2 + i]);
  }
#pragma unroll
  for (int i = 0; i < HD / 32; ++i) {
    float v0[4], v1[4];
    mm_lds4(sv + mm_value<float, HD>(2 * tig, 8 * i + gid), v0);
    mm_lds4(sv + mm_value<float, HD>(2 * tig + 1, 8 * i + gid), v1);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t h0, l0, h1, l1;
      mm_split(v0[k], h0, l0);
      mm_split(v1[k], h1, l1);
      float y[4] = {};
      mma_tf32_1688(y, pl, h0, h1);
      mma_tf32_1688(y, ph, l0, l1);
      mma_tf32_1688(y, ph, h0, h1);
#pragma unroll
      for (int e = 0; e < 4; ++e) x.o[4 * i + k][e] += y[e];
    }
  }
}

template <typename T, int HD>
__global__ void __launch_bounds__(MM_THREADS, MmCfg<T, HD>::CTAS)
    paged_mma_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedWork w) {
  using C = MmCfg<T, HD>;
  auto ex2 = [](float v) { return sizeof(T) == 4 ? exp2f(v) : ex2_fast(v); };
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float s_m[MM_WARPS][MM_ROWS], s_l[MM_WARPS][MM_ROWS];
  float* join = reinterpret_cast<float*>(smem + MM_WARPS * C::RING);  // [warps][MM_JOIN]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int gid = lane >> 2, tig = lane & 3;
  const uint32_t ring = smem_u32(smem) + warp * C::RING;
  pdl_trigger();
  pdl_wait();
  __shared__ PagedSpan told;
  PagedSpan span;
  if (!paged_plan<MM_ROWS, C::BLOCK>(a, w, told, span)) return;
  PagedSpan ls = span;
  PagedPart p;
  bool have = paged_next<MM_ROWS, C::BLOCK>(a, w, span, p);
  if (!have) return;  // no block of an item, its lead alone
  const T* q = static_cast<const T*>(a.q);

  // the tile to load next; its page number is looked at when it is loaded, a tile later
  PagedPart lp;
  const int32_t* row = nullptr;
  int lb = 0, lpage = 0;
  bool more = true;
  auto find = [&](bool next_part) {
    if (next_part) {
      more = paged_next<MM_ROWS, C::BLOCK>(a, w, ls, lp);  // (there is a first one)
      lb = lp.b0;
      row = paged_row(a, lp);
    }
    const int k0 = lb * C::BLOCK + C::KEYS * warp;
    if (more && k0 < lp.x.keys) lpage = row[k0 >> a.page_shift];
  };
  auto load = [&](int stage) {
    if (more) {
      const int k0 = lb * C::BLOCK + C::KEYS * warp, keys = lp.x.keys - k0;
      if (keys > 0) {
        const size_t at = paged_at<HD>(a, paged_sound(a, lpage), lp.h, k0);
        mm_load_tile<T, HD>(a, ring + stage * (2 * C::TILE), at, keys);
      }
      ++lb;
      find(lb >= lp.b1);
    }
    cp_async_commit();
  };
  MmRows<T, HD> x;
  auto load_q = [&]() {
    const int r0 = p.r * MM_ROWS + gid;
    const bool in0 = r0 < p.x.rows, in1 = r0 + 8 < p.x.rows;
    mm_load_q<HD>(x, q + (in0 ? paged_q_at<HD>(a, p, r0) : 0), q + (in1 ? paged_q_at<HD>(a, p, r0 + 8) : 0), in0, in1);
  };
  find(true);
  load_q();
#pragma unroll
  for (int i = 0; i < MM_STAGES - 1; ++i) load(i);

  int use = 0, fill = MM_STAGES - 1;  // stages
  while (have) {
    const int rows = min(MM_ROWS, p.x.rows - p.r * MM_ROWS), all = p.x.keys, b1 = p.b1, slot = p.slot;
    mm_clear<T, HD>(x);
    for (int b = p.b0; b < b1; ++b) {
      load(fill);
      cp_async_wait<MM_STAGES - 1>();
      __syncwarp();
      const int keys = all - (b * C::BLOCK + C::KEYS * warp);
      if (keys > 0) mm_tile<HD>(x, ring + use * (2 * C::TILE), keys, a.scale_log2);
      __syncwarp();  // the stage is read: the next load may fill it
      use = use + 1 == MM_STAGES ? 0 : use + 1;
      fill = fill + 1 == MM_STAGES ? 0 : fill + 1;
    }
    // the next part's queries are on their way while this one's results are joined
    have = paged_next<MM_ROWS, C::BLOCK>(a, w, span, p);
    if (have) load_q();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x.l[i] += __shfl_xor_sync(0xffffffffu, x.l[i], 1);
      x.l[i] += __shfl_xor_sync(0xffffffffu, x.l[i], 2);
      if (tig == 0) {
        s_m[warp][gid + 8 * i] = x.m[i];
        s_l[warp][gid + 8 * i] = x.l[i];
      }
    }
    // The part's result from the four warps', all dims at once for up to 8 rows (more rows
    // of 128 dims: half of the dims at a time)
    const int dims = rows > 8 ? min(64, HD) : HD;
    for (int d0 = 0; d0 < HD; d0 += dims) {
      float* j0 = join + warp * MM_JOIN + gid * dims;
      mm_put<HD>(x, j0, j0 + 8 * dims, d0, dims, gid < rows, gid + 8 < rows);
      __syncthreads();
      const int quads = dims / 4;
      for (int i = tid; i < rows * quads; i += MM_THREADS) {
        const int r = i / quads, c = (i - r * quads) * 4;
        float top = s_m[0][r];
#pragma unroll
        for (int k = 1; k < MM_WARPS; ++k) top = fmaxf(top, s_m[k][r]);
        const float base = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < MM_WARPS; ++k) {
          const float f = ex2(s_m[k][r] - base);
          const float4 y = *reinterpret_cast<const float4*>(join + k * MM_JOIN + r * dims + (c ^ ((r & 3) * 8)));
          sum = fmaf(f, s_l[k][r], sum);
          z.x = fmaf(f, y.x, z.x), z.y = fmaf(f, y.y, z.y), z.z = fmaf(f, y.z, z.z), z.w = fmaf(f, y.w, z.w);
        }
        const float inv = sum > 0.f ? 1.f / sum : sum;  // (NaN stays NaN)
        const size_t at = static_cast<size_t>(slot) * MM_ROWS + r;
        *reinterpret_cast<float4*>(w.o + at * HD + d0 + c) = make_float4(z.x * inv, z.y * inv, z.z * inv, z.w * inv);
        if (d0 + c == 0) w.lse2[at] = top + log2f(sum);
      }
      __syncthreads();  // the buffer and the warps' maxima and sums are read
    }
  }
  cp_async_wait<0>();
}

// A CTA of W warps has up to 16 rows of a sequence and KV head over all that they see,
// prefix and own entries one after the other, and writes the results: no plan, no partial
// results, one launch.  The prefix is read once for every sequence, in L2.
// PARTS: the prefixes' partial results are in w already (the 128-row tiles'), and this
// launch has the sequences' own entries and joins.
template <typename T, int HD, int W, int R, bool PARTS>
__global__ void __launch_bounds__(32 * W, 8 / W)
    paged_direct_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedWork w) {
  using C = MmCfg<T, HD>;
  constexpr int LOG = C::KEYS == 16 ? 4 : 3;
  auto ex2 = [](float v) { return sizeof(T) == 4 ? exp2f(v) : ex2_fast(v); };
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float s_m[W][MM_ROWS], s_l[W][MM_ROWS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  const uint32_t ring = smem_u32(smem) + warp * C::RING;
  const int s = static_cast<int>(blockIdx.x), n_rows = a.n_q * a.per, tiles = (n_rows + MM_ROWS - 1) / MM_ROWS;
  const int g = static_cast<int>(blockIdx.y) / tiles, r0 = (static_cast<int>(blockIdx.y) - g * tiles) * MM_ROWS;
  const int rows = min(MM_ROWS, n_rows - r0);
  pdl_trigger();
  pdl_wait();
  MmRows<T, HD> x;
  auto q_row = [&](int r) {  // row r of the sequence and KV head
    const size_t tok = static_cast<size_t>(s) * a.n_q + r / a.per;
    return static_cast<const T*>(a.q) + (tok * (static_cast<size_t>(a.Hkv) * a.per) + static_cast<size_t>(g) * a.per + r % a.per) * HD;
  };
  const bool in0 = gid < rows, in1 = gid + 8 < rows;
  mm_load_q<HD>(x, q_row(in0 ? r0 + gid : 0), q_row(in1 ? r0 + gid + 8 : 0), in0, in1);
  mm_clear<T, HD>(x);
  const int own = max(0, paged_len(a.lens[s], a.cols << a.page_shift) - (a.n_q - 1));
  const int32_t *shared_row = nullptr, *own_row = a.table + static_cast<size_t>(s) * a.cols;
  int shared = 0, per = 0;
  PagedGroup e{};
  if (PARTS) {
    per = w.head[0];
    e = paged_group_of(a, s, w.head + 1);
    if (e.g < 0) return;  // a row behind the last sequence stays as it was
  } else if (a.G > 0) {
    e = paged_group_of(a, s, nullptr);
    if (e.g < 0) return;
    if (threadIdx.x == 0 && e.beyond) atomicOr(a.status, kStatusBadIndex);
    shared = e.keys;
    shared_row = a.ptable + static_cast<size_t>(e.g) * a.pcols;
  }
  // tiles of keys, those of the prefix first: warp w has w, w + W, ...; the pages of
  // its next 32 tiles are asked for together
  const int n_shared = (shared + C::KEYS - 1) >> LOG, n = n_shared + ((own + C::KEYS - 1) >> LOG), mine = n > warp ? (n - warp + W - 1) / W : 0;
  int pages = 0;
  auto load = [&](int i) {  // the warp's i-th tile into stage i % MM_STAGES
    if (i < mine) {
      if ((i & 31) == 0) {
        const int t = warp + W * (i + lane);
        pages = t < n_shared ? shared_row[t << LOG >> a.page_shift] : t < n ? own_row[(t - n_shared) << LOG >> a.page_shift] : 0;
      }
      const int t = warp + W * i, k0 = (t < n_shared ? t : t - n_shared) << LOG;
      const int page = paged_sound(a, __shfl_sync(0xffffffffu, pages, i & 31));
      mm_load_tile<T, HD>(a, ring + i % MM_STAGES * (2 * C::TILE), paged_at<HD>(a, page, g, k0), (t < n_shared ? shared : own) - k0);
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < MM_STAGES - 1; ++i) load(i);
  for (int i = 0; i < mine; ++i) {
    load(i + MM_STAGES - 1);
    cp_async_wait<MM_STAGES - 1>();
    __syncwarp();
    const int t = warp + W * i;
    mm_tile<HD>(x, ring + i % MM_STAGES * (2 * C::TILE), t < n_shared ? shared - (t << LOG) : own - ((t - n_shared) << LOG), a.scale_log2);
    __syncwarp();  // the stage is read: the next load may fill it
  }
  cp_async_wait<0>();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x.l[i] += __shfl_xor_sync(0xffffffffu, x.l[i], 1);
    x.l[i] += __shfl_xor_sync(0xffffffffu, x.l[i], 2);
    if (tig == 0) {
      s_m[warp][gid + 8 * i] = x.m[i];
      s_l[warp][gid + 8 * i] = x.l[i];
    }
  }
  // the warps' results in the ring's place
  __syncthreads();
  float* join = reinterpret_cast<float*>(smem);  // [W][rows][HD]
  float* j0 = join + (warp * MM_ROWS + gid) * HD;
  mm_put<HD>(x, j0, j0 + 8 * HD, 0, HD, in0, in1);
  __syncthreads();
  constexpr int DPL = HD / 32;
  PagedRows<HD, R> y;  // (rows warp, warp + W, ...: R W rows or fewer)
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = warp + i * W;
    y.rr[i] = r < rows ? r0 + r : -1;
    y.m[i] = s_m[0][r];
#pragma unroll
    for (int k = 1; k < W; ++k) y.m[i] = fmaxf(y.m[i], s_m[k][r]);
    const float base = y.m[i] == -INFINITY ? 0.f : y.m[i];
    y.l[i] = 0.f;
#pragma unroll
    for (int d = 0; d < DPL; ++d) y.acc[i][d] = 0.f;
    if (r >= rows) continue;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const float f = ex2(s_m[k][r] - base);
      const float* z = join + (k * MM_ROWS + r) * HD + ((lane * DPL) ^ ((r & 3) * 8));
      y.l[i] = fmaf(f, s_l[k][r], y.l[i]);
#pragma unroll
      for (int d = 0; d < DPL; ++d) y.acc[i][d] = fmaf(f, z[d], y.acc[i][d]);
    }
  }
  if (PARTS) {
    JoinParts pre[R], none[R] = {};
#pragma unroll
    for (int i = 0; i < R; ++i)
      pre[i] = y.rr[i] < 0 ? JoinParts{nullptr, nullptr, 0, 0} : join_prefix(a, w, e, per, s, g, y.rr[i], HD);
    paged_add_parts<T, HD, R, 16 / R>(y, pre, none);
  }
  paged_finish<T, HD, R>(a, s, g, y);
}

}  // namespace

template <typename T, int HD>
static cudaError_t run_mma(const PagedArgs& a, const PagedWork& w, int ctas, cudaStream_t s) {
  static OncePerDevice once;
  const cudaError_t e = set_smem_limit_once(once, paged_mma_kernel<T, HD>, MmCfg<T, HD>::SMEM);
  if (e != cudaSuccess) return e;
  ZSAA_LAUNCH(paged_mma_kernel<T, HD>, dim3(ctas), dim3(MM_THREADS), MmCfg<T, HD>::SMEM, s, a, w);
  return cudaSuccess;
}

template <typename T, int HD, int W, int R, bool PARTS>
static cudaError_t run_direct(const PagedArgs& a, const PagedWork& w, cudaStream_t s) {
  static OncePerDevice once;
  const int smem = std::max(W * MmCfg<T, HD>::RING, W * MM_ROWS * HD * 4);  // (the ring, then the warps' results)
  const cudaError_t e = set_smem_limit_once(once, paged_direct_kernel<T, HD, W, R, PARTS>, smem);
  if (e != cudaSuccess) return e;
  const int tiles = (a.n_q * a.per + MM_ROWS - 1) / MM_ROWS;
  ZSAA_LAUNCH(paged_direct_kernel<T, HD, W, R, PARTS>, dim3(a.S, a.Hkv * tiles), dim3(32 * W), smem, s, a, w);
  return cudaSuccess;
}

// R: the rows that a warp finishes together.  With 4 rows to a head (us, R of 4 and of 1): 64
// sequences of 600 entries after a prefix of 32000, 128 dims, 93.1 and 86.4; of 150 after 16000,
// 64 dims, 35.8 and 30.9: a row that is not there still takes its turns in the reductions.
template <typename T, int HD, int W, bool PARTS>
static cudaError_t run_direct(const PagedArgs& a, const PagedWork& w, cudaStream_t s) {
  constexpr int FEW = W == 2 ? 2 : 1;
  if (a.n_q * a.per <= FEW * W) return run_direct<T, HD, W, FEW, PARTS>(a, w, s);
  return run_direct<T, HD, W, MM_ROWS / W, PARTS>(a, w, s);
}

// Warps of a CTA: eight where CTAs of four would leave SMs empty, two where more than two of
// four would be asked of an SM, so that one's start and end run under the others' loads (us,
// four and two, 64 sequences, 8 heads of 128 dims: 32 keys 6.1 and 3.9, 256 17.0 and 14.4, 512
// 27.3 and 24.7, float32 8.2 and 6.5, 34 and 31, 58 and 55; 64 dims 4.8 and 3.7, 8.3 and 8.8, 18
// and 16; 62 of 5 queries, 256 keys 32 and 27, 64 dims 18 and 19; 30 of one 6.2 and 9.2).  Four
// after partial results: with 600 own entries after 16000, 128 dims, 64 sequences 61 and 59, 30
// 38 and 45; 24 of 4 drafts 22 and 28.
template <typename T, int HD>
static cudaError_t run_direct(const PagedArgs& a, const PagedWork* w, cudaStream_t s) {
  const long long ctas = static_cast<long long>(a.S) * a.Hkv * ((a.n_q * a.per + MM_ROWS - 1) / MM_ROWS);
  if constexpr (sizeof(T) == 2)
    if (w != nullptr) return ctas <= 152 ? run_direct<T, HD, 8, true>(a, *w, s) : run_direct<T, HD, 4, true>(a, *w, s);
  if (ctas <= 152) return run_direct<T, HD, 8, false>(a, PagedWork{}, s);
  return ctas <= 304 ? run_direct<T, HD, 4, false>(a, PagedWork{}, s) : run_direct<T, HD, 2, false>(a, PagedWork{}, s);
}

// Lead: without, with 2 and with 8 units to an item (us): 60 sequences of 160 entries on 57
// prefixes of 850 to 1700, 128 dims, 79, 64 and 66, float32 189, 149 and 171; 62 sequences of 5
// queries on one prefix of 1024, float32, 356, 174 and 209; 32 in 8 groups, prefix 1204, 20, 20
// and 24.
PagedTiles paged_mma_tiles(int dtype, int hd, int sms) {
  const bool bf = dtype == ZSAA_BF16;
  const int ctas = hd == 128 ? MmCfg<bf16, 128>::CTAS : hd == 64 ? MmCfg<bf16, 64>::CTAS : MmCfg<float, 32>::CTAS;
  return PagedTiles{MM_ROWS, bf ? MmCfg<bf16, 128>::BLOCK : MmCfg<float, 128>::BLOCK, ctas * sms, 1, 2};
}

cudaError_t launch_paged_direct(const PagedArgs& a, const PagedWork* prefixes, int dtype, int hd, cudaStream_t s) {
  if (dtype == ZSAA_BF16) return hd == 64 ? run_direct<bf16, 64>(a, prefixes, s) : run_direct<bf16, 128>(a, prefixes, s);
  if (hd == 32) return run_direct<float, 32>(a, nullptr, s);
  return hd == 64 ? run_direct<float, 64>(a, nullptr, s) : run_direct<float, 128>(a, nullptr, s);
}

cudaError_t launch_paged_mma(const PagedArgs& a, const PagedWork& w, int dtype, int hd, int ctas, cudaStream_t s) {
  if (dtype == ZSAA_BF16) return hd == 64 ? run_mma<bf16, 64>(a, w, ctas, s) : run_mma<bf16, 128>(a, w, ctas, s);
  if (hd == 32) return run_mma<float, 32>(a, w, ctas, s);
  return hd == 64 ? run_mma<float, 64>(a, w, ctas, s) : run_mma<float, 128>(a, w, ctas, s);
}

}  // namespace zsaa
