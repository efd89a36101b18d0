// Attention over a paged cache for few query rows (bf16): tiles of 16 rows against the
// keys of an entry on mma.sync m16n8k16.
//
// A decode step has n_q * (Hq / Hkv) rows to each KV head, 4 or 8 as a rule, so the
// keys and values stream past once and the tensor work is small: the kernel is bound
// by HBM on long caches and by its chain of loads on short ones.  Each of the 4 warps
// walks its own 16 keys of every block of 64 with a ring of cp.async stages of its own,
// so nothing but the end of a part synchronises the CTA; 16 keys never leave a page.
// The ring runs ahead over the ends of parts: a CTA with several short items has the
// next item's keys in flight while it joins its warps' results of the last.
//
// Per 16 keys: S = Q K^T, the running maximum (moved only when the tile's exceeds it by
// 2^8: P entries up to 256 are exact in float32 and in the pair), P = 2^(S scale - m)
// carried as the bf16 pair P_hi + P_lo (one bf16 would cost 0.1% in every output), and
// O += P_hi V + P_lo V in float32.
#include "paged.cuh"

namespace zsaa {
namespace {

constexpr int MM_WARPS = 4, MM_THREADS = 32 * MM_WARPS, MM_ROWS = 16, MM_KEYS = 16 * MM_WARPS;
constexpr int MM_STAGES = 3;
constexpr int MM_JOIN = 1024;  // floats of a warp in the buffer that joins results: 8 rows of 128 dims, 16 of 64
constexpr float MM_RESCALE_LOG2 = 8.f;

template <int HD>
struct MmCfg {
  static constexpr int TILE = 16 * HD * 2;  // 16 keys, or their values
  static constexpr int RING = MM_STAGES * 2 * TILE;  // a warp's
  static constexpr int JOIN = MM_WARPS * MM_JOIN * 4;
  static constexpr int SMEM = MM_WARPS * RING + JOIN;
  static constexpr int CTAS = HD == 128 ? 2 : 3;  // resident per SM
};

// byte offset of 16-byte chunk c of row r, chunks XOR-swizzled by the row (conflict-free ldmatrix)
template <int HD>
__device__ __forceinline__ uint32_t mm_swz(int r, int c) {
  return static_cast<uint32_t>(r * HD * 2 + ((c ^ (r & 7)) << 4));
}

// A warp's rows: queries as the A operand (rows gid and gid + 8, dims 2 tig, 2 tig + 1 and
// those + 8 of every 16), accumulators, and maximum and sum of rows gid and gid + 8 (the sum
// of this thread's keys alone).
template <int HD>
struct MmRows {
  uint32_t q[HD / 16][4];
  float o[HD / 8][4];
  float m[2], l[2];
};
template <int HD>
__device__ __forceinline__ void mm_clear(MmRows<HD>& x) {
#pragma unroll
  for (int i = 0; i < HD / 8; ++i) x.o[i][0] = x.o[i][1] = x.o[i][2] = x.o[i][3] = 0.f;
  x.m[0] = x.m[1] = -INFINITY;
  x.l[0] = x.l[1] = 0.f;
}
// q0, q1: rows gid and gid + 8; in0, in1: whether there are such
template <int HD>
__device__ __forceinline__ void mm_load_q(MmRows<HD>& x, const bf16* q0, const bf16* q1, bool in0, bool in1) {
  const int tig = threadIdx.x & 3;
#pragma unroll
  for (int kk = 0; kk < HD / 16; ++kk) {
    x.q[kk][0] = in0 ? *reinterpret_cast<const uint32_t*>(q0 + 16 * kk + 2 * tig) : 0u;
    x.q[kk][1] = in1 ? *reinterpret_cast<const uint32_t*>(q1 + 16 * kk + 2 * tig) : 0u;
    x.q[kk][2] = in0 ? *reinterpret_cast<const uint32_t*>(q0 + 16 * kk + 8 + 2 * tig) : 0u;
    x.q[kk][3] = in1 ? *reinterpret_cast<const uint32_t*>(q1 + 16 * kk + 8 + 2 * tig) : 0u;
  }
}
// Asks for up to 16 keys and their values, which lie one after the other from element `at`
// on; rows past `keys` are zero.
template <int HD>
__device__ __forceinline__ void mm_load_tile(const PagedArgs& a, uint32_t sk, size_t at, int keys) {
  constexpr int CH = HD / 8, STEP = 32 / CH;  // chunks per row, rows per round
  const int lane = threadIdx.x & 31, c = lane % CH;
  const uint32_t sv = sk + MmCfg<HD>::TILE;
#pragma unroll
  for (int i = 0; i < 16 / STEP; ++i) {
    const int r = lane / CH + i * STEP;
    const size_t from = at + static_cast<size_t>(r < keys ? r : 0) * HD + c * 8;
    cp_async16(sk + mm_swz<HD>(r, c), static_cast<const bf16*>(a.k) + from, r < keys);
    cp_async16(sv + mm_swz<HD>(r, c), static_cast<const bf16*>(a.v) + from, r < keys);
  }
}
// 16 keys (the first `keys` count) and their values at sk
template <int HD>
__device__ __forceinline__ void mm_tile(MmRows<HD>& x, uint32_t sk, int keys, float scale) {
  const int lane = threadIdx.x & 31, tig = lane & 3, mi = lane >> 3;
  const uint32_t sv = sk + MmCfg<HD>::TILE;
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

template <int HD>
__global__ void __launch_bounds__(MM_THREADS, MmCfg<HD>::CTAS)
    paged_mma_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedWork w) {
  using C = MmCfg<HD>;
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
  if (!paged_plan<MM_ROWS, MM_KEYS>(a, w, told, span)) return;
  const bf16* q = static_cast<const bf16*>(a.q);

  // the tile to load next; its page number is looked at when it is loaded, a tile later
  PagedSpan ls = span;
  PagedPart lp;
  const int32_t* row = nullptr;
  int lb = 0, lpage = 0;
  bool more = true;
  auto find = [&](bool next_part) {
    if (next_part) {
      more = paged_next<MM_ROWS, MM_KEYS>(a, w, ls, lp);
      lb = lp.b0;
      row = paged_row(a, lp);
    }
    const int k0 = lb * MM_KEYS + 16 * warp;
    if (more && k0 < lp.x.keys) lpage = row[k0 >> a.page_shift];
  };
  auto load = [&](int stage) {
    if (more) {
      const int k0 = lb * MM_KEYS + 16 * warp, keys = lp.x.keys - k0;
      if (keys > 0) {
        const size_t at = paged_at<HD>(a, paged_sound(a, lpage), lp.h, k0);
        mm_load_tile<HD>(a, ring + stage * (2 * C::TILE), at, keys);
      }
      ++lb;
      find(lb >= lp.b1);
    }
    cp_async_commit();
  };
  PagedPart p;
  bool have = paged_next<MM_ROWS, MM_KEYS>(a, w, span, p);
  MmRows<HD> x;
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
    mm_clear<HD>(x);
    for (int b = p.b0; b < b1; ++b) {
      load(fill);
      cp_async_wait<MM_STAGES - 1>();
      __syncwarp();
      const int keys = all - (b * MM_KEYS + 16 * warp);
      if (keys > 0) mm_tile<HD>(x, ring + use * (2 * C::TILE), keys, a.scale_log2);
      __syncwarp();  // the stage is read: the next load may fill it
      use = use + 1 == MM_STAGES ? 0 : use + 1;
      fill = fill + 1 == MM_STAGES ? 0 : fill + 1;
    }
    // the next part's queries are on their way while this one's results are joined
    have = paged_next<MM_ROWS, MM_KEYS>(a, w, span, p);
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
    // of 128 dims: half of the dims at a time).  A row's groups of 8 floats are XORed by its
    // number, which keeps stores and loads clear of bank conflicts.
    const int dims = rows > 8 ? min(64, HD) : HD;
    for (int d0 = 0; d0 < HD; d0 += dims) {
#pragma unroll
      for (int i = 0; i < HD / 8; ++i)
        if (8 * i >= d0 && 8 * i < d0 + dims) {
          float* j0 = join + warp * MM_JOIN + gid * dims + ((8 * i - d0) ^ ((gid & 3) * 8)) + 2 * tig;
          if (gid < rows) *reinterpret_cast<float2*>(j0) = make_float2(x.o[i][0], x.o[i][1]);
          if (gid + 8 < rows) *reinterpret_cast<float2*>(j0 + 8 * dims) = make_float2(x.o[i][2], x.o[i][3]);
        }
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
          const float f = ex2_fast(s_m[k][r] - base);
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
template <int HD, int W, bool PARTS>
__global__ void __launch_bounds__(32 * W, 8 / W)
    paged_direct_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedWork w) {
  using C = MmCfg<HD>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float s_m[W][MM_ROWS], s_l[W][MM_ROWS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
  const uint32_t ring = smem_u32(smem) + warp * C::RING;
  const int s = static_cast<int>(blockIdx.x), n_rows = a.n_q * a.per, tiles = (n_rows + MM_ROWS - 1) / MM_ROWS;
  const int g = static_cast<int>(blockIdx.y) / tiles, r0 = (static_cast<int>(blockIdx.y) - g * tiles) * MM_ROWS;
  const int rows = min(MM_ROWS, n_rows - r0);
  pdl_trigger();
  pdl_wait();
  MmRows<HD> x;
  auto q_row = [&](int r) {  // row r of the sequence and KV head
    const size_t tok = static_cast<size_t>(s) * a.n_q + r / a.per;
    return static_cast<const bf16*>(a.q) + (tok * (static_cast<size_t>(a.Hkv) * a.per) + static_cast<size_t>(g) * a.per + r % a.per) * HD;
  };
  const bool in0 = gid < rows, in1 = gid + 8 < rows;
  mm_load_q<HD>(x, q_row(in0 ? r0 + gid : 0), q_row(in1 ? r0 + gid + 8 : 0), in0, in1);
  mm_clear<HD>(x);
  const int own = max(0, min(a.lens[s], a.cols << a.page_shift) - (a.n_q - 1));
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
  // tiles of 16 keys, those of the prefix first: warp w has w, w + W, ...; the pages of
  // its next 32 tiles are asked for together
  const int n_shared = (shared + 15) >> 4, n = n_shared + ((own + 15) >> 4), mine = n > warp ? (n - warp + W - 1) / W : 0;
  int pages = 0;
  auto load = [&](int i) {  // the warp's i-th tile into stage i % MM_STAGES
    if (i < mine) {
      if ((i & 31) == 0) {
        const int t = warp + W * (i + lane);
        pages = t < n_shared ? shared_row[t << 4 >> a.page_shift] : t < n ? own_row[(t - n_shared) << 4 >> a.page_shift] : 0;
      }
      const int t = warp + W * i, k0 = (t < n_shared ? t : t - n_shared) << 4;
      const int page = paged_sound(a, __shfl_sync(0xffffffffu, pages, i & 31));
      mm_load_tile<HD>(a, ring + i % MM_STAGES * (2 * C::TILE), paged_at<HD>(a, page, g, k0), (t < n_shared ? shared : own) - k0);
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
    mm_tile<HD>(x, ring + i % MM_STAGES * (2 * C::TILE), t < n_shared ? shared - (t << 4) : own - ((t - n_shared) << 4), a.scale_log2);
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
  // the warps' results in the ring's place, a row's groups of 8 floats XORed by its number
  __syncthreads();
  float* join = reinterpret_cast<float*>(smem);  // [W][rows][HD]
#pragma unroll
  for (int i = 0; i < HD / 8; ++i) {
    float* j0 = join + (warp * MM_ROWS + gid) * HD + ((8 * i) ^ ((gid & 3) * 8)) + 2 * tig;
    if (in0) *reinterpret_cast<float2*>(j0) = make_float2(x.o[i][0], x.o[i][1]);
    if (in1) *reinterpret_cast<float2*>(j0 + 8 * HD) = make_float2(x.o[i][2], x.o[i][3]);
  }
  __syncthreads();
  constexpr int DPL = HD / 32;
  constexpr int R = MM_ROWS / W;
  PagedRows<HD, R> y;
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
      const float f = ex2_fast(s_m[k][r] - base);
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
    paged_add_parts<bf16, HD, R, 16 / R>(y, pre, none);
  }
  paged_finish<bf16, HD, R>(a, s, g, y);
}

}  // namespace

PagedTiles paged_mma_tiles(int hd, int sms) {
  return PagedTiles{MM_ROWS, MM_KEYS, (hd == 128 ? MmCfg<128>::CTAS : MmCfg<64>::CTAS) * sms, 1};
}

template <int HD>
static cudaError_t run_mma(const PagedArgs& a, const PagedWork& w, int ctas, cudaStream_t s) {
  static OncePerDevice once;
  const cudaError_t e = set_smem_limit_once(once, paged_mma_kernel<HD>, MmCfg<HD>::SMEM);
  if (e != cudaSuccess) return e;
  ZSAA_LAUNCH(paged_mma_kernel<HD>, dim3(ctas), dim3(MM_THREADS), MmCfg<HD>::SMEM, s, a, w);
  return cudaSuccess;
}

template <int HD, int W, bool PARTS>
static cudaError_t run_direct(const PagedArgs& a, const PagedWork& w, cudaStream_t s) {
  static OncePerDevice once;
  const cudaError_t e = set_smem_limit_once(once, paged_direct_kernel<HD, W, PARTS>, W * MmCfg<HD>::RING);
  if (e != cudaSuccess) return e;
  const int tiles = (a.n_q * a.per + MM_ROWS - 1) / MM_ROWS;
  ZSAA_LAUNCH(paged_direct_kernel<HD, W, PARTS>, dim3(a.S, a.Hkv * tiles), dim3(32 * W), W * MmCfg<HD>::RING, s, a, w);
  return cudaSuccess;
}

cudaError_t launch_paged_direct(const PagedArgs& a, const PagedWork* prefixes, int hd, bool wide, cudaStream_t s) {
  const PagedWork w = prefixes != nullptr ? *prefixes : PagedWork{};
  if (prefixes != nullptr) {
    if (hd == 64) return wide ? run_direct<64, 8, true>(a, w, s) : run_direct<64, 4, true>(a, w, s);
    return wide ? run_direct<128, 8, true>(a, w, s) : run_direct<128, 4, true>(a, w, s);
  }
  if (hd == 64) return wide ? run_direct<64, 8, false>(a, w, s) : run_direct<64, 4, false>(a, w, s);
  return wide ? run_direct<128, 8, false>(a, w, s) : run_direct<128, 4, false>(a, w, s);
}

cudaError_t launch_paged_mma(const PagedArgs& a, const PagedWork& w, int hd, int ctas, cudaStream_t s) {
  return hd == 64 ? run_mma<64>(a, w, ctas, s) : run_mma<128>(a, w, ctas, s);
}

}  // namespace zsaa
