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

template <int HD>
__global__ void __launch_bounds__(MM_THREADS, MmCfg<HD>::CTAS)
    paged_mma_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedWork w) {
  using C = MmCfg<HD>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float s_m[MM_WARPS][MM_ROWS], s_l[MM_WARPS][MM_ROWS];
  float* join = reinterpret_cast<float*>(smem + MM_WARPS * C::RING);  // [warps][MM_JOIN]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int gid = lane >> 2, tig = lane & 3, mi = lane >> 3;
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
        const uint32_t sk = ring + stage * (2 * C::TILE), sv = sk + C::TILE;
        constexpr int CH = HD / 8, STEP = 32 / CH;  // chunks per row, rows per round
        const int c = lane % CH;
#pragma unroll
        for (int i = 0; i < 16 / STEP; ++i) {
          const int r = lane / CH + i * STEP;
          const size_t from = at + static_cast<size_t>(r < keys ? r : 0) * HD + c * 8;
          cp_async16(sk + mm_swz<HD>(r, c), static_cast<const bf16*>(a.k) + from, r < keys);
          cp_async16(sv + mm_swz<HD>(r, c), static_cast<const bf16*>(a.v) + from, r < keys);
        }
      }
      ++lb;
      find(lb >= lp.b1);
    }
    cp_async_commit();
  };
  PagedPart p;
  bool have = paged_next<MM_ROWS, MM_KEYS>(a, w, span, p);
  // Q as the A operand: rows gid and gid + 8, dims 2 tig, 2 tig + 1 and those + 8
  uint32_t qf[HD / 16][4];
  auto load_q = [&]() {
    const int r0 = p.r * MM_ROWS + gid;
    const bool in0 = r0 < p.x.rows, in1 = r0 + 8 < p.x.rows;
    const bf16* q0 = q + (in0 ? paged_q_at<HD>(a, p, r0) : 0) + 2 * tig;
    const bf16* q1 = q + (in1 ? paged_q_at<HD>(a, p, r0 + 8) : 0) + 2 * tig;
#pragma unroll
    for (int kk = 0; kk < HD / 16; ++kk) {
      qf[kk][0] = in0 ? *reinterpret_cast<const uint32_t*>(q0 + 16 * kk) : 0u;
      qf[kk][1] = in1 ? *reinterpret_cast<const uint32_t*>(q1 + 16 * kk) : 0u;
      qf[kk][2] = in0 ? *reinterpret_cast<const uint32_t*>(q0 + 16 * kk + 8) : 0u;
      qf[kk][3] = in1 ? *reinterpret_cast<const uint32_t*>(q1 + 16 * kk + 8) : 0u;
    }
  };
  find(true);
  load_q();
#pragma unroll
  for (int i = 0; i < MM_STAGES - 1; ++i) load(i);

  int use = 0, fill = MM_STAGES - 1;  // stages
  while (have) {
    const int rows = min(MM_ROWS, p.x.rows - p.r * MM_ROWS), all = p.x.keys, b1 = p.b1, slot = p.slot;
    float o[HD / 8][4];
#pragma unroll
    for (int i = 0; i < HD / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};  // of rows gid, gid + 8; l of this thread's keys
    for (int b = p.b0; b < b1; ++b) {
      load(fill);
      cp_async_wait<MM_STAGES - 1>();
      __syncwarp();
      const int keys = all - (b * MM_KEYS + 16 * warp);
      if (keys > 0) {
        const uint32_t sk = ring + use * (2 * C::TILE), sv = sk + C::TILE;
        float s[2][4] = {};
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
          uint32_t b0, b1, b2, b3;
          ldsm_x4(sk + mm_swz<HD>((mi >> 1) * 8 + (lane & 7), kk * 2 + (mi & 1)), b0, b1, b2, b3);
          mma_bf16_16816(s[0], qf[kk], b0, b1);
          mma_bf16_16816(s[1], qf[kk], b2, b3);
        }
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[t][e] = 8 * t + 2 * tig + (e & 1) < keys ? s[t][e] * a.scale_log2 : -INFINITY;
            mx[e >> 1] = fmaxf(mx[e >> 1], s[t][e]);
          }
        bool need = false;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
          mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
          need |= mx[i] > m[i] + MM_RESCALE_LOG2;
        }
        if (__any_sync(0xffffffffu, need)) {
          float f[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float mn = fmaxf(m[i], mx[i]);
            f[i] = mn == -INFINITY ? 1.f : ex2_fast(m[i] - mn);
            m[i] = mn;
            l[i] *= f[i];
          }
#pragma unroll
          for (int i = 0; i < HD / 8; ++i) {
            o[i][0] *= f[0];
            o[i][1] *= f[0];
            o[i][2] *= f[1];
            o[i][3] *= f[1];
          }
        }
        const float base[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float p0 = ex2_fast(s[t][2 * i] - base[i]), p1 = ex2_fast(s[t][2 * i + 1] - base[i]);
            l[i] += p0 + p1;
            const uint32_t u = pack_bf16x2(p0, p1);
            hi[2 * t + i] = u;
            lo[2 * t + i] = pack_bf16x2(p0 - bf16lo(u), p1 - bf16hi(u));
          }
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) {
          uint32_t b0, b1, b2, b3;
          ldsm_x4_t(sv + mm_swz<HD>((mi & 1) * 8 + (lane & 7), d * 2 + (mi >> 1)), b0, b1, b2, b3);
          mma_bf16_16816(o[2 * d], hi, b0, b1);
          mma_bf16_16816(o[2 * d + 1], hi, b2, b3);
          mma_bf16_16816(o[2 * d], lo, b0, b1);
          mma_bf16_16816(o[2 * d + 1], lo, b2, b3);
        }
      }
      __syncwarp();  // the stage is read: the next load may fill it
      use = use + 1 == MM_STAGES ? 0 : use + 1;
      fill = fill + 1 == MM_STAGES ? 0 : fill + 1;
    }
    // the next part's queries are on their way while this one's results are joined
    have = paged_next<MM_ROWS, MM_KEYS>(a, w, span, p);
    if (have) load_q();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
      if (tig == 0) {
        s_m[warp][gid + 8 * i] = m[i];
        s_l[warp][gid + 8 * i] = l[i];
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
          if (gid < rows) *reinterpret_cast<float2*>(j0) = make_float2(o[i][0], o[i][1]);
          if (gid + 8 < rows) *reinterpret_cast<float2*>(j0 + 8 * dims) = make_float2(o[i][2], o[i][3]);
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
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < MM_WARPS; ++k) {
          const float f = ex2_fast(s_m[k][r] - base);
          const float4 y = *reinterpret_cast<const float4*>(join + k * MM_JOIN + r * dims + (c ^ ((r & 3) * 8)));
          sum = fmaf(f, s_l[k][r], sum);
          x.x = fmaf(f, y.x, x.x), x.y = fmaf(f, y.y, x.y), x.z = fmaf(f, y.z, x.z), x.w = fmaf(f, y.w, x.w);
        }
        const float inv = sum > 0.f ? 1.f / sum : sum;  // (NaN stays NaN)
        const size_t at = static_cast<size_t>(slot) * MM_ROWS + r;
        *reinterpret_cast<float4*>(w.o + at * HD + d0 + c) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
        if (d0 + c == 0) w.lse2[at] = top + log2f(sum);
      }
      __syncthreads();  // the buffer and the warps' maxima and sums are read
    }
  }
  cp_async_wait<0>();
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

cudaError_t launch_paged_mma(const PagedArgs& a, const PagedWork& w, int hd, int ctas, cudaStream_t s) {
  return hd == 64 ? run_mma<64>(a, w, ctas, s) : run_mma<128>(a, w, ctas, s);
}

}  // namespace zsaa
