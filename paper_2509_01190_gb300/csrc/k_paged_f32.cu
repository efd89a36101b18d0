// Attention over a paged cache in float32, on the CUDA cores: tiles of 16 query rows against
// blocks of 32 keys in shared memory, online softmax (log2 domain) in 32 bits.  The next
// block's keys and values are on their way to registers while one is worked on.  Bound by the chain of a block's steps (scores, softmax,
// P V), with one CTA on an SM 1.2 us at 32 dims and 2.5 at 128; page numbers fetched a block
// ahead took registers and gained nothing (40 and 40 us for 1024 keys of 32 dims, 53 and 67
// with 64).
#include "paged.cuh"

namespace zsaa {
namespace {

constexpr int F_THREADS = 128, F_ROWS = 16, F_KEYS = 32;

template <int HD>
struct FCfg {
  static constexpr int LD = HD + 4;
  static constexpr int QUADS = HD / 4, GROUPS = F_THREADS / QUADS, RPG = F_ROWS / GROUPS;  // P V: 4 dims of RPG rows a thread
  static constexpr int NL = F_KEYS * (HD / 8) / F_THREADS;  // 8-dim pieces of a block's keys that a thread loads
};

template <int HD>
struct FShared {
  float q[F_ROWS][FCfg<HD>::LD], k[F_KEYS][FCfg<HD>::LD], v[F_KEYS][HD];
  float p[F_KEYS][F_ROWS + 4];  // probabilities, by key: a thread's rows of P V lie together
  float s[F_ROWS][F_KEYS + 4], corr[F_ROWS], l[F_ROWS], m[F_ROWS];
};

template <int HD>
struct FRows {
  float m, l;  // of row tid / 8, the same in its 8 threads
  float acc[FCfg<HD>::RPG][4];
};
template <int HD>
__device__ __forceinline__ void f_clear(FRows<HD>& x) {
  x.m = -INFINITY;
  x.l = 0.f;
#pragma unroll
  for (int i = 0; i < FCfg<HD>::RPG; ++i) x.acc[i][0] = x.acc[i][1] = x.acc[i][2] = x.acc[i][3] = 0.f;
}

__device__ __forceinline__ void f_load8(const float* p, float (&x)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

// rows of queries, element offset `at(r)` of row r; rows past the tile's are zero
template <int HD, typename At>
__device__ __forceinline__ void f_load_q(const PagedArgs& a, FShared<HD>& sh, int rows, At at) {
  for (int i = threadIdx.x; i < F_ROWS * (HD / 8); i += F_THREADS) {
    const int r = i / (HD / 8), c = (i % (HD / 8)) * 8;
    float x[8] = {};
    if (r < rows) f_load8(static_cast<const float*>(a.q) + at(r) + c, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) sh.q[r][c + j] = x[j];
  }
}

// Keys [k0, k1) of a table row and KV head h.  All threads.
template <int HD>
__device__ __forceinline__ void f_keys(const PagedArgs& a, FShared<HD>& sh, FRows<HD>& x, const int32_t* table, int h, int k0,
                                       int k1) {
  using C = FCfg<HD>;
  const int tid = threadIdx.x;
  const int ty = tid >> 4, tx = tid & 15;       // scores: rows 2 ty, 2 ty + 1, keys tx, tx + 16
  const int sr = tid >> 3, sc = (tid & 7) * 4;  // softmax: row, first of 4 keys
  const int quad = (tid % C::QUADS) * 4, rg = tid / C::QUADS;
  float kx[C::NL][8], vx[C::NL][8];
  auto fetch = [&](int k) {
#pragma unroll
    for (int i = 0; i < C::NL; ++i) {
      const int e = tid + i * F_THREADS, r = k + e / (HD / 8), c = (e % (HD / 8)) * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) kx[i][j] = vx[i][j] = 0.f;
      if (r < k1) {
        const size_t at = paged_at<HD>(a, paged_page(a, table, r), h, r) + c;
        f_load8(static_cast<const float*>(a.k) + at, kx[i]);
        f_load8(static_cast<const float*>(a.v) + at, vx[i]);
      }
    }
  };
  if (k0 < k1) fetch(k0);
  for (int k = k0; k < k1; k += F_KEYS) {
    const int keys = min(F_KEYS, k1 - k);
#pragma unroll
    for (int i = 0; i < C::NL; ++i) {
      const int e = tid + i * F_THREADS, r = e / (HD / 8), c = (e % (HD / 8)) * 8;
#pragma unroll
      for (int j = 0; j < 8; j += 4) {
        *reinterpret_cast<float4*>(&sh.k[r][c + j]) = make_float4(kx[i][j], kx[i][j + 1], kx[i][j + 2], kx[i][j + 3]);
        *reinterpret_cast<float4*>(&sh.v[r][c + j]) = make_float4(vx[i][j], vx[i][j + 1], vx[i][j + 2], vx[i][j + 3]);
      }
    }
    __syncthreads();
    if (k + F_KEYS < k1) fetch(k + F_KEYS);
    float s[2][2] = {};
#pragma unroll 8
    for (int c = 0; c < HD; c += 4) {
      const float4 q0 = *reinterpret_cast<const float4*>(&sh.q[2 * ty][c]);
      const float4 q1 = *reinterpret_cast<const float4*>(&sh.q[2 * ty + 1][c]);
      const float4 y0 = *reinterpret_cast<const float4*>(&sh.k[tx][c]);
      const float4 y1 = *reinterpret_cast<const float4*>(&sh.k[tx + 16][c]);
      auto dot = [](const float4& u, const float4& v, float z) {
        return fmaf(u.w, v.w, fmaf(u.z, v.z, fmaf(u.y, v.y, fmaf(u.x, v.x, z))));
      };
      s[0][0] = dot(q0, y0, s[0][0]);
      s[0][1] = dot(q0, y1, s[0][1]);
      s[1][0] = dot(q1, y0, s[1][0]);
      s[1][1] = dot(q1, y1, s[1][1]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) sh.s[2 * ty + i][tx + 16 * j] = tx + 16 * j < keys ? s[i][j] * a.scale_log2 : -INFINITY;
    __syncthreads();
    const float4 v4 = *reinterpret_cast<const float4*>(&sh.s[sr][sc]);
    float v[4] = {v4.x, v4.y, v4.z, v4.w}, mx = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    const float mn = fmaxf(x.m, mx), base = mn == -INFINITY ? 0.f : mn;
    const float corr = exp2f(x.m - base);
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = exp2f(v[j] - base);
      sum += v[j];
      sh.p[sc + j][sr] = v[j];
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    x.l = x.l * corr + sum;
    x.m = mn;
    if ((tid & 7) == 0) sh.corr[sr] = corr;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < C::RPG; ++i) {
      const float f = sh.corr[rg * C::RPG + i];
#pragma unroll
      for (int j = 0; j < 4; ++j) x.acc[i][j] *= f;
    }
#pragma unroll 8
    for (int e = 0; e < F_KEYS; ++e) {  // (past the last key both factors are 0)
      const float4 y = *reinterpret_cast<const float4*>(&sh.v[e][quad]);
      float p[C::RPG];
      if constexpr (C::RPG == 4) {
        const float4 u = *reinterpret_cast<const float4*>(&sh.p[e][rg * 4]);
        p[0] = u.x, p[1] = u.y, p[2] = u.z, p[3] = u.w;
      } else {
#pragma unroll
        for (int i = 0; i < C::RPG; ++i) p[i] = sh.p[e][rg * C::RPG + i];
      }
#pragma unroll
      for (int i = 0; i < C::RPG; ++i) {
        x.acc[i][0] = fmaf(p[i], y.x, x.acc[i][0]);
        x.acc[i][1] = fmaf(p[i], y.y, x.acc[i][1]);
        x.acc[i][2] = fmaf(p[i], y.z, x.acc[i][2]);
        x.acc[i][3] = fmaf(p[i], y.w, x.acc[i][3]);
      }
    }
    __syncthreads();  // the block is read
  }
  if ((tid & 7) == 0) {
    sh.l[sr] = x.l;
    sh.m[sr] = x.m;
  }
}

template <int HD>
__global__ void __launch_bounds__(F_THREADS)
    paged_f32_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedWork w) {
  using C = FCfg<HD>;
  __shared__ __align__(16) FShared<HD> sh;
  __shared__ PagedSpan told;
  const int quad = (threadIdx.x % C::QUADS) * 4, rg = threadIdx.x / C::QUADS;
  pdl_trigger();
  pdl_wait();
  PagedSpan span;
  if (!paged_plan<F_ROWS, F_KEYS>(a, w, told, span)) return;
  PagedPart p;
  while (paged_next<F_ROWS, F_KEYS>(a, w, span, p)) {
    const int rows = min(F_ROWS, p.x.rows - p.r * F_ROWS);
    __syncthreads();  // the part before is done with shared memory
    f_load_q<HD>(a, sh, rows, [&](int r) { return paged_q_at<HD>(a, p, p.r * F_ROWS + r); });
    FRows<HD> x;
    f_clear<HD>(x);
    f_keys<HD>(a, sh, x, paged_row(a, p), p.h, p.b0 * F_KEYS, min(p.b1 * F_KEYS, p.x.keys));
    __syncthreads();
#pragma unroll
    for (int i = 0; i < C::RPG; ++i) {
      const int r = rg * C::RPG + i;
      if (r >= rows) continue;
      const float inv = sh.l[r] > 0.f ? 1.f / sh.l[r] : sh.l[r];  // (NaN stays NaN)
      float* o = w.o + (static_cast<size_t>(p.slot) * F_ROWS + r) * HD + quad;
      *reinterpret_cast<float4*>(o) = make_float4(x.acc[i][0] * inv, x.acc[i][1] * inv, x.acc[i][2] * inv, x.acc[i][3] * inv);
      if (quad == 0) w.lse2[static_cast<size_t>(p.slot) * F_ROWS + r] = sh.m[r] + log2f(sh.l[r]);
    }
  }
}

// Short calls: up to 16 rows of a sequence and KV head over all that they see, prefix and
// own entries one after the other, and the results: no plan, no partial results, one launch.
template <int HD>
__global__ void __launch_bounds__(F_THREADS) paged_f32_direct_kernel(const __grid_constant__ PagedArgs a) {
  using C = FCfg<HD>;
  __shared__ __align__(16) FShared<HD> sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int quad = (threadIdx.x % C::QUADS) * 4, rg = threadIdx.x / C::QUADS;
  const int s = static_cast<int>(blockIdx.x), n_rows = a.n_q * a.per, tiles = (n_rows + F_ROWS - 1) / F_ROWS;
  const int g = static_cast<int>(blockIdx.y) / tiles, r0 = (static_cast<int>(blockIdx.y) - g * tiles) * F_ROWS;
  const int rows = min(F_ROWS, n_rows - r0);
  pdl_trigger();
  pdl_wait();
  FRows<HD> x;
  f_clear<HD>(x);
  f_load_q<HD>(a, sh, rows, [&](int r) {
    const size_t tok = static_cast<size_t>(s) * a.n_q + (r0 + r) / a.per;
    return (tok * (static_cast<size_t>(a.Hkv) * a.per) + static_cast<size_t>(g) * a.per + (r0 + r) % a.per) * HD;
  });
  const int own = max(0, min(a.lens[s], a.cols << a.page_shift) - (a.n_q - 1));
  if (a.G > 0) {
    const PagedGroup e = paged_group_of(a, s, nullptr);
    if (e.g < 0) return;  // a row behind the last sequence stays as it was
    if (threadIdx.x == 0 && e.beyond) atomicOr(a.status, kStatusBadIndex);
    f_keys<HD>(a, sh, x, a.ptable + static_cast<size_t>(e.g) * a.pcols, g, 0, e.keys);
  }
  f_keys<HD>(a, sh, x, a.table + static_cast<size_t>(s) * a.cols, g, 0, own);
#pragma unroll
  for (int i = 0; i < C::RPG; ++i)
    *reinterpret_cast<float4*>(&sh.k[rg * C::RPG + i][quad]) = make_float4(x.acc[i][0], x.acc[i][1], x.acc[i][2], x.acc[i][3]);
  __syncthreads();
  constexpr int DPL = HD / 32;
  constexpr int W = F_THREADS / 32, R = F_ROWS / W;
  PagedRows<HD, R> y;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = warp + i * W;
    y.rr[i] = r < rows ? r0 + r : -1;
    y.m[i] = sh.m[r];
    y.l[i] = sh.l[r];
#pragma unroll
    for (int d = 0; d < DPL; ++d) y.acc[i][d] = sh.k[r][lane * DPL + d];
  }
  paged_finish<float, HD, R>(a, s, g, y);
}

template <int HD>
cudaError_t run_f32(const PagedArgs& a, const PagedWork* w, int ctas, cudaStream_t s) {
  if (w != nullptr) {
    ZSAA_LAUNCH(paged_f32_kernel<HD>, dim3(ctas), dim3(F_THREADS), 0, s, a, *w);
  } else {
    const int tiles = (a.n_q * a.per + F_ROWS - 1) / F_ROWS;
    ZSAA_LAUNCH(paged_f32_direct_kernel<HD>, dim3(a.S, a.Hkv * tiles), dim3(F_THREADS), 0, s, a);
  }
  return cudaSuccess;
}
cudaError_t launch(const PagedArgs& a, const PagedWork* w, int hd, int ctas, cudaStream_t s) {
  if (hd == 32) return run_f32<32>(a, w, ctas, s);
  return hd == 64 ? run_f32<64>(a, w, ctas, s) : run_f32<128>(a, w, ctas, s);
}

}  // namespace

PagedTiles paged_f32_tiles(int sms) { return PagedTiles{F_ROWS, F_KEYS, 4 * sms, 1}; }

cudaError_t launch_paged_f32(const PagedArgs& a, const PagedWork& w, int hd, int ctas, cudaStream_t s) {
  return launch(a, &w, hd, ctas, s);
}
cudaError_t launch_paged_f32_direct(const PagedArgs& a, int hd, cudaStream_t s) { return launch(a, nullptr, hd, 0, s); }

}  // namespace zsaa
