// Attention over a paged cache for many query rows (bf16) on the sm_103a tensor cores:
// tiles of 128 rows against the keys of an entry, as a shared prefix has them (the rows
// of a KV head are the queries of all sequences that share it).
//
// Per block of 128 keys, with one accumulating tile per CTA and two CTAs per SM:
//   S = Q K^T             (tcgen05, 128 x 128 x hd; K's pages by TMA, 128-byte swizzle)
//   softmax warps         (one query row per thread, TMEM lane = row): row maximum, moved
//                         only when the block's exceeds it by 2^8; P = 2^(S scale - m) as
//                         the bf16 pair P_hi + P_lo over S's columns, the sum in float32
//   O += P_hi V + P_lo V  (A = P from TMEM, B = V as it lies in its pages, MN-major)
// While one CTA's softmax runs, the other's products do.  Tensor work for a block is
// 1.0 us at the measured rate however few of the 128 rows are in use, its keys and values
// (64 KB) take 1.4 us of an SM's share of HBM, which the tiles of a prefix share in L2.  Beyond
// 128 rows to a prefix neither is the bound: with 256 rows to a head and a prefix of 32000 (58
// us) the tensor pipe is active for 38% of the cycles and HBM gives 2.3 TB/s, while the thread
// that issues is busy for 83%: a switch between the operand forms of S (A from shared memory)
// and of P V (A from TMEM) costs the pipe some 500 clocks.
//
// Roles (192 threads): warp 0 TMA producer (K and V in rings of their own, a lane per
// page), warp 1 MMA issuer, warps 2-5 softmax, Q and results (warp w has TMEM lanes
// 32 (w % 4) .. + 31).  Order of the tensor work: S(0) | PV(0) S(1) | PV(1) S(2) ...;
// tcgen05.mma executes in issue order, so S(j+1) overwrites P(j) after it is read, and S(j)
// being complete says that PV(j-1) is.  At the end of a part the next part's Q is loaded
// before this one's results are read out, so its first S runs under that.  Every wait is
// bounded; after one that ran out every role stops, copies in flight are drained, and
// TMEM is freed.
#include "kernels.h"
#include "paged.cuh"

namespace zsaa {
namespace {

constexpr int TC_ROWS = 128, TC_KEYS = 128;
constexpr int TC_THREADS = 192;
constexpr uint32_t TC_TMEM_COLS = 256;  // S (then P) in 0-127, O from 128 on
constexpr uint32_t TC_O_COL = 128;
constexpr float TC_RESCALE_LOG2 = 8.f;

template <int HD>
struct TcCfg {
  static constexpr int CH = HD / 64;            // 64-dim (128-byte) chunks
  static constexpr int TILE = TC_ROWS * HD * 2;  // Q, a block of K, or one of V
  static constexpr int STAGES = HD == 128 ? 1 : 2;
  static constexpr int SMEM = TILE * (1 + 2 * STAGES) + 256 + 1024;
};

// Shared-memory descriptor of an MN-major operand with the 128-byte swizzle: rows of 64
// bf16 along N for consecutive K, 8-row atoms 1024 B apart along K, 64-element chunks
// along N `chunk` bytes apart.
__device__ __forceinline__ uint64_t tc_desc_mn(uint32_t saddr, uint32_t chunk) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | static_cast<uint64_t>((chunk >> 4) & 0x3FFFu) << 16 |
         static_cast<uint64_t>(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

// D[tmem] (+)= A[tmem] B[smem]: A's rows are the lanes, two bf16 of K to a column
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u)
      : "memory");
}

// maximum of three in one instruction
__device__ __forceinline__ float tc_max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

__device__ __forceinline__ void tc_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

template <int HD>
__global__ void __launch_bounds__(TC_THREADS, 2)
    paged_tc_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                    const __grid_constant__ PagedArgs a, const __grid_constant__ PagedWork w) {
  using C = TcCfg<HD>;
  constexpr int CH = C::CH, TILE = C::TILE, ST = C::STAGES, CHUNK = TC_KEYS * 128;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t *sQ = smem, *sK = sQ + TILE, *sV = sK + ST * TILE;
  uint64_t* bars = reinterpret_cast<uint64_t*>(sV + ST * TILE);
  uint64_t *q_full = bars, *s_full = bars + 1, *p_full = bars + 2, *o_full = bars + 3, *mma_done = bars + 4;
  uint64_t *k_full = bars + 5, *k_empty = k_full + ST, *v_full = k_empty + ST, *v_empty = v_full + ST;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(v_empty + ST);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(q_full, 4);
    mbar_init(s_full, 1);
    mbar_init(p_full, 4);
    mbar_init(o_full, 1);
    mbar_init(mma_done, 1);
    for (int i = 0; i < ST; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 1);
      mbar_init(&v_full[i], 1);
      mbar_init(&v_empty[i], 1);
    }
    *abort_flag = 0;
    fence_barrier_init();
    prefetch_tmap(&tm_k);
    prefetch_tmap(&tm_v);
  }
  // TMEM is taken between the wait and the trigger.  An allocation blocks: columns taken before
  // the wait could be those that a CTA of the kernel before still waits for, and a kernel let
  // in before the allocation could take those that this one's CTAs need, and then wait for them.
  pdl_wait();
  if (warp == 1) tmem_alloc(tmem_slot, TC_TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_trigger();

  __shared__ PagedSpan told;
  PagedSpan span;
  const bool work = paged_plan<TC_ROWS, TC_KEYS>(a, w, told, span);
  PagedPart p;
  if (work && warp == 0) {
    // ---------------------------------------------------------------- TMA producer
    bool ok = true;
    uint32_t J = 0;  // blocks asked for
    const int box = min(1 << a.page_shift, TC_KEYS);  // rows of a copy
    bool k_sent = false;
    while (ok && paged_next<TC_ROWS, TC_KEYS>(a, w, span, p)) {
      const int32_t* table = paged_row(a, p);
      for (int b = p.b0; b < p.b1; ++b, ++J) {
        const int k0 = b * TC_KEYS, n = (min(TC_KEYS, p.x.keys - k0) + box - 1) / box;
        int row = 0;  // of this lane's copy, in the pool
        if (lane < n) {
          const int i = k0 + lane * box;
          row = ((paged_page(a, table, i) * a.Hkv + p.h) << a.page_shift) + (i & ((1 << a.page_shift) - 1));
        }
        const uint32_t st = J % ST, turn = ((J / ST) & 1) ^ 1;
        auto send = [&](const CUtensorMap* tm, uint8_t* to, uint64_t* full, uint64_t* empty) {
          if (!__all_sync(0xffffffffu, mbar_wait_ab(&empty[st], turn, a.status, abort_flag))) return false;
          if (lane == 0) mbar_arrive_expect_tx(&full[st], n * box * HD * 2);
          __syncwarp();
          if (lane < n)
            for (int c = 0; c < CH; ++c)
              tma_load_2d(to + st * TILE + c * CHUNK + lane * box * 128, tm, c * 64, row, &full[st]);
          return true;
        };
        ok = send(&tm_k, sK, k_full, k_empty);
        if (!ok) break;
        k_sent = true;
        ok = send(&tm_v, sV, v_full, v_empty);
        if (!ok) break;
        k_sent = false;
      }
    }
    if (!ok && lane == 0) {  // let the copies already asked for land before the CTA's memory goes away
      const uint32_t nk = J + (k_sent ? 1 : 0);
      for (uint32_t k = nk; k > 0 && k + ST > nk; --k) mbar_wait(&k_full[(k - 1) % ST], ((k - 1) / ST) & 1, nullptr);
      for (uint32_t k = J; k > 0 && k + ST > J; --k) mbar_wait(&v_full[(k - 1) % ST], ((k - 1) / ST) & 1, nullptr);
    }
    __syncwarp();
  } else if (work && warp == 1) {
    // ---------------------------------------------------------------- MMA issuer
    if (lane == 0) {
      bool ok = true;
      uint32_t J = 0, parts = 0;
      auto issue_s = [&](uint32_t j, int keys) {
        if (!mbar_wait_ab(&k_full[j % ST], (j / ST) & 1, a.status, abort_flag)) return false;
        tc_fence_after();
        const uint32_t idesc = idesc_bf16_f32(TC_ROWS, (keys + 15) & ~15), q = smem_u32(sQ), k = smem_u32(sK + (j % ST) * TILE);
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk)
          tc_mma_bf16(tmem, sdesc_sw128(q + (kk / 4) * CHUNK + (kk % 4) * 32), sdesc_sw128(k + (kk / 4) * CHUNK + (kk % 4) * 32),
                      idesc, kk > 0 ? 1u : 0u);
        tc_commit(s_full);
        tc_commit(&k_empty[j % ST]);
        return true;
      };
      auto issue_pv = [&](uint32_t j, int keys, bool first) {
        if (!mbar_wait_ab(&v_full[j % ST], (j / ST) & 1, a.status, abort_flag) ||
            !mbar_wait_ab(p_full, j & 1, a.status, abort_flag))
          return false;
        tc_fence_after();
        constexpr uint32_t idesc = idesc_bf16_f32(TC_ROWS, HD) | (1u << 16);  // B (V) MN-major
        const uint32_t v = smem_u32(sV + (j % ST) * TILE);
        for (int kk = 0; kk < (keys + 15) / 16; ++kk)
#pragma unroll
          for (int part = 0; part < 2; ++part)
            tc_mma_ts(tmem + TC_O_COL, tmem + 32 * (kk / 2) + 16 * part + 8 * (kk % 2),
                      tc_desc_mn(v + kk * 16 * 128, HD > 64 ? CHUNK : 1024), idesc, !(first && kk == 0 && part == 0));
        tc_commit(&v_empty[j % ST]);
        return true;
      };
      while (ok && paged_next<TC_ROWS, TC_KEYS>(a, w, span, p)) {
        auto keys = [&](int b) { return min(TC_KEYS, p.x.keys - b * TC_KEYS); };
        ok = mbar_wait_ab(q_full, parts & 1, a.status, abort_flag) && issue_s(J, keys(p.b0));
        for (int b = p.b0; ok && b < p.b1; ++b, ++J) {
          ok = issue_pv(J, keys(b), b == p.b0);
          if (!ok) break;
          if (b + 1 < p.b1)
            ok = issue_s(J + 1, keys(b + 1));
          else
            tc_commit(o_full);
        }
        ++parts;
      }
      // every MMA issued has finished before the CTA frees TMEM
      if (parts > 0) {
        tc_commit(mma_done);
        mbar_wait(mma_done, 0, a.status);
      }
    }
    __syncwarp();
  } else if (work) {
    // ---------------------------------------------------------------- softmax, Q, results
    const int quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
    const uint32_t s_addr = tmem + lanes, o_addr = tmem + lanes + TC_O_COL;
    const bf16* q = static_cast<const bf16*>(a.q);
    bool ok = true;
    uint32_t J = 0, parts = 0;
    auto arrive = [&](uint64_t* bar) {
      __syncwarp();
      if (lane == 0) tc_arrive(bar);
    };
    // the tile's rows into shared memory, as the S products read them; rows past the entry's are zero
    auto load_q = [&]() {
      const int rr = p.r * TC_ROWS + row;
      const bool live = rr < p.x.rows;
      const uint4* src = reinterpret_cast<const uint4*>(q + (live ? paged_q_at<HD>(a, p, rr) : 0));
      uint4 x[HD / 8];
#pragma unroll
      for (int u = 0; u < HD / 8; ++u) x[u] = live ? src[u] : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int u = 0; u < HD / 8; ++u)
        *reinterpret_cast<uint4*>(sQ + (u / 8) * CHUNK + row * 128 + (((u % 8) ^ (row & 7)) << 4)) = x[u];
      fence_proxy_async_smem();
      arrive(q_full);
    };
    bool have = paged_next<TC_ROWS, TC_KEYS>(a, w, span, p);
    if (have) load_q();
    while (have) {
      const int rows = min(TC_ROWS, p.x.rows - p.r * TC_ROWS), keys_all = p.x.keys, b0 = p.b0, b1 = p.b1, slot = p.slot;
      const bool mine = quad * 32 < rows;  // some row of the warp is a query
      float m = -INFINITY, l = 0.f;
      for (int b = b0; b < b1; ++b, ++J) {
        const int keys = min(TC_KEYS, keys_all - b * TC_KEYS), n_ch = (keys + 31) / 32;
        ok = ok && __all_sync(0xffffffffu, mbar_wait_ab(s_full, J & 1, a.status, abort_flag));
        tc_fence_after();
        if (keys & 15) {
          // P is zero past the last key, but V's rows there are whatever its page holds:
          // keep one that is not finite out of 0 * V
          ok = ok && __all_sync(0xffffffffu, mbar_wait_ab(&v_full[J % ST], (J / ST) & 1, a.status, abort_flag));
          const uint32_t va = smem_u32(sV + (J % ST) * TILE);
          const int per = (-keys & 15) * 8;
          for (int i = row; i < per * CH; i += TC_ROWS)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(va + (i / per) * CHUNK + keys * 128 + (i % per) * 16), "r"(0)
                         : "memory");
          fence_proxy_async_smem();
        }
        if (ok && mine) {
          auto hide = [&](uint32_t (&v)[32], int c) {  // columns past the last key
            if (32 * c + 32 > keys) {
#pragma unroll
              for (int e = 0; e < 32; ++e) v[e] = 32 * c + e < keys ? v[e] : 0xff800000u;
            }
          };
          float mx = -INFINITY;
#pragma unroll 1
          for (int c = 0; c < n_ch; ++c) {
            uint32_t v[32];
            tmem_ld32(s_addr + 32 * c, v);
            tmem_ld_wait();
            hide(v, c);
            float m4[4] = {mx, mx, mx, mx};
#pragma unroll
            for (int e = 0; e < 32; e += 8)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                m4[k] = tc_max3(m4[k], __uint_as_float(v[e + 2 * k]), __uint_as_float(v[e + 2 * k + 1]));
            mx = fmaxf(tc_max3(m4[0], m4[1], m4[2]), m4[3]);
          }
          const float mb = mx == -INFINITY ? -INFINITY : mx * a.scale_log2;
          const bool need = mb > m + TC_RESCALE_LOG2;
          if (__any_sync(0xffffffffu, need)) {
            const float mn = need ? mb : m;
            const float f = need ? (m == -INFINITY ? 0.f : ex2_fast(m - mn)) : 1.f;
            if (b > b0) {  // O holds the part's blocks before this one
#pragma unroll 1
              for (int c = 0; c < HD / 32; ++c) {
                uint32_t v[32];
                tmem_ld32(o_addr + 32 * c, v);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * f);
                tmem_st16(o_addr + 32 * c, *reinterpret_cast<const uint32_t(*)[16]>(v));
                tmem_st16(o_addr + 32 * c + 16, *reinterpret_cast<const uint32_t(*)[16]>(v + 16));
              }
            }
            l *= f;
            m = mn;
          }
          // P over the columns just read; the next chunk's load is in flight meanwhile
          const float base = m == -INFINITY ? 0.f : m;
          const uint64_t scale2 = f2pack(a.scale_log2, a.scale_log2), nm2 = f2pack(-base, -base);
          uint32_t v[32];
          tmem_ld32(s_addr, v);
          tmem_ld_wait();
#pragma unroll 1
          for (int c = 0; c < n_ch; ++c) {
            hide(v, c);
            uint64_t t[16];
#pragma unroll
            for (int e = 0; e < 16; ++e)
              t[e] = ffma2(f2pack(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])), scale2, nm2);
            if (c + 1 < n_ch) tmem_ld32(s_addr + 32 * (c + 1), v);
            uint32_t hi[16], lo[16];
            uint64_t sum = f2pack(0.f, 0.f);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float p0, p1, r0, r1;
              f2unpack(t[e], p0, p1);
              const uint64_t pp = f2pack(ex2_fast(p0), ex2_fast(p1));
              sum = fadd2(sum, pp);
              f2unpack(pp, p0, p1);
              hi[e] = pack_bf16x2(p0, p1);
              f2unpack(fsub2(pp, f2pack(bf16lo(hi[e]), bf16hi(hi[e]))), r0, r1);
              lo[e] = pack_bf16x2(r0, r1);
            }
            float l0, l1;
            f2unpack(sum, l0, l1);
            l += l0 + l1;
            tmem_st16(s_addr + 32 * c, hi);
            tmem_st16(s_addr + 32 * c + 16, lo);
            tmem_ld_wait();
          }
          tmem_st_wait();
        }
        tc_fence_before();
        arrive(p_full);
      }
      // the next part's Q (every S of this one is complete), then this one's results
      have = paged_next<TC_ROWS, TC_KEYS>(a, w, span, p);
      if (have) load_q();
      ok = ok && __all_sync(0xffffffffu, mbar_wait_ab(o_full, parts & 1, a.status, abort_flag));
      ++parts;
      tc_fence_after();
      if (ok && mine) {
        const float inv = l > 0.f ? 1.f / l : l;  // (NaN stays NaN)
        const size_t at = static_cast<size_t>(slot) * TC_ROWS + row;
        float* o = w.o + at * HD;
#pragma unroll 1
        for (int c = 0; c < HD / 32; ++c) {
          uint32_t v[32];
          tmem_ld32(o_addr + 32 * c, v);
          tmem_ld_wait();
          if (row < rows) {
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * inv);
#pragma unroll
            for (int e = 0; e < 32; e += 8) st_global_v8(o + 32 * c + e, v + e);
          }
        }
        if (row < rows) w.lse2[at] = m + log2f(l);
      }
      tc_fence_before();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, TC_TMEM_COLS);
  }
}

bool encode_pool(CUtensorMap* m, const void* base, int hd, uint64_t rows, int box) {
  EncodeTiledFn enc = get_encode_tiled();
  if (enc == nullptr) return false;
  cuuint64_t dims[2] = {static_cast<cuuint64_t>(hd), rows};
  cuuint64_t strides[1] = {static_cast<cuuint64_t>(hd) * 2};
  cuuint32_t size[2] = {64, static_cast<cuuint32_t>(box)};
  cuuint32_t es[2] = {1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, size, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD>
cudaError_t run_tc(const PagedArgs& a, const PagedWork& w, int ctas, cudaStream_t s) {
  static OncePerDevice once;
  const cudaError_t e = set_smem_limit_once(once, paged_tc_kernel<HD>, TcCfg<HD>::SMEM);
  if (e != cudaSuccess) return e;
  const uint64_t rows = (static_cast<uint64_t>(a.n_pages) * a.Hkv) << a.page_shift;
  const int box = 1 << a.page_shift < TC_KEYS ? 1 << a.page_shift : TC_KEYS;
  CUtensorMap tk, tv;
  if (!encode_pool(&tk, a.k, HD, rows, box) || !encode_pool(&tv, a.v, HD, rows, box)) return cudaErrorInvalidValue;
  ZSAA_LAUNCH(paged_tc_kernel<HD>, dim3(ctas), dim3(TC_THREADS), TcCfg<HD>::SMEM, s, tk, tv, a, w);
  return cudaSuccess;
}

}  // namespace

// Lead: with 0, 1 and 4 units to an item (us): 128 sequences in 20 groups of 3000, 64 dims, 52, 53
// and 55; 64 dims and 24 sequences in 6 groups of 1500, 31, 30 and 32; a prefix of 32000, 128
// dims, 96, 93 and 92.
PagedTiles paged_tc_tiles(int sms) { return PagedTiles{TC_ROWS, TC_KEYS, 2 * sms, 2, 1}; }

cudaError_t launch_paged_tc(const PagedArgs& a, const PagedWork& w, int hd, int ctas, cudaStream_t s) {
  return hd == 64 ? run_tc<64>(a, w, ctas, s) : run_tc<128>(a, w, ctas, s);
}

}  // namespace zsaa
