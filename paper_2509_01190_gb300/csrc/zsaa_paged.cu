// C ABI of the paged-cache and beam-search calls: argument checks and launches.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "common.cuh"
#include "paged.h"

namespace zsaa {
void set_last_error(const char* msg);
}

using namespace zsaa;

namespace {

zsaa_status refuse(zsaa_status st, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  set_last_error(buf);
  return st;
}
zsaa_status bad(const char* msg) { return refuse(ZSAA_ERR_INVALID_ARG, "%s", msg); }

#define ZTRY(expr)                              \
  do {                                          \
    const zsaa_status st_ = (expr);             \
    if (st_ != ZSAA_OK) return st_;             \
  } while (0)

zsaa_status launched(const char* call, cudaError_t e) {
  if (e == cudaSuccess) return ZSAA_OK;
  return refuse(ZSAA_ERR_CUDA, "%s: launch failed: %s", call, cudaGetErrorString(e));
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
// int32 and float32 arrays (or null)
template <typename... P>
bool words(const P*... p) {
  return ((reinterpret_cast<uintptr_t>(p) | ...) & 3) == 0;
}
bool overlap(const void* a, size_t an, const void* b, size_t bn) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + bn && y < x + an;
}

constexpr long long kMostInt = 0x7fffffff;

size_t element(int dtype) { return dtype == ZSAA_BF16 ? 2 : 4; }

zsaa_status check_pages(const zsaa_pages* kv) {
  if (kv == nullptr) return bad("null pages");
  if (kv->dtype != ZSAA_F32 && kv->dtype != ZSAA_BF16) return bad("bad dtype");
  if (kv->n_pages < 1 || kv->n_kv_heads < 1) return bad("n_pages and n_kv_heads must be >= 1");
  const int p = kv->page_size;
  if (p < 16 || p > 256 || (p & (p - 1)) != 0)
    return refuse(ZSAA_ERR_UNSUPPORTED, "page_size %d is not 16, 32, 64, 128 or 256", p);
  if (kv->head_dim != 64 && kv->head_dim != 128 && !(kv->head_dim == 32 && kv->dtype == ZSAA_F32))
    return refuse(ZSAA_ERR_UNSUPPORTED, "paged caches need head_dim 64 or 128 (float32: or 32)");
  if (static_cast<long long>(kv->n_pages) * kv->n_kv_heads > kMostInt / p)
    return bad("n_pages * n_kv_heads * page_size must be below 2^31");
  return ZSAA_OK;
}
zsaa_status check_pool(const zsaa_pages* kv) {
  if (kv->k == nullptr || kv->v == nullptr) return bad("null pool");
  if (!aligned(kv->k, 16) || !aligned(kv->v, 16)) return bad("pools must be 16-byte aligned");
  return ZSAA_OK;
}
zsaa_status check_cols(int cols, int page) {
  if (cols < 1 || cols > kMostInt / page) return bad("a table row needs 1 or more pages, and below 2^31 entries");
  return ZSAA_OK;
}
int page_shift(int page) {
  int n = 0;
  while ((1 << n) < page) ++n;
  return n;
}

zsaa_status device_sms(int* sms) {
  static OncePerDevice once;
  static int found[64] = {};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess)
    e = once.run([&] { return cudaDeviceGetAttribute(&found[dev], cudaDevAttrMultiProcessorCount, dev); });
  if (e != cudaSuccess) return refuse(ZSAA_ERR_CUDA, "no usable current device (%s)", cudaGetErrorString(e));
  *sms = found[dev];
  return ZSAA_OK;
}
zsaa_status status_word(int** w) {
  *w = shared_status_word();
  return *w != nullptr ? ZSAA_OK : refuse(ZSAA_ERR_CUDA, "status word allocation failed");
}

// sizes of an attention call, without its pointers
zsaa_status attention_sizes(const zsaa_pages* kv, int S, int n_q, int Hq, int G, int cols, int prefix_cols,
                            PagedArgs* a, size_t* bytes) {
  ZTRY(check_pages(kv));
  if (S < 1 || Hq < 1) return bad("S and Hq must be >= 1");
  if (n_q < 1 || n_q > 16) return refuse(ZSAA_ERR_UNSUPPORTED, "n_q=%d outside [1, 16]", n_q);
  if (Hq % kv->n_kv_heads != 0) return bad("Hq must be a multiple of n_kv_heads");
  if (Hq > 65536) return bad("more than 65536 heads");  // (a grid's second dimension)
  if (G < 0) return bad("G must be >= 0");
  ZTRY(check_cols(cols, kv->page_size));
  if (G > 0) ZTRY(check_cols(prefix_cols, kv->page_size));
  // (the kernels round a row's entries up to blocks of keys, the largest of 128)
  if (cols > (kMostInt - 255) / kv->page_size || (G > 0 && prefix_cols > (kMostInt - 255) / kv->page_size))
    return bad("a table row of an attention call holds at most 2^31 - 256 entries");
  if (static_cast<long long>(S) * n_q > kMostInt / 32 / Hq || G > kMostInt / 2 - S)
    return bad("too many query rows or groups");
  *a = PagedArgs{};
  a->n_pages = kv->n_pages;
  a->page_shift = page_shift(kv->page_size);
  a->Hkv = kv->n_kv_heads;
  a->per = Hq / kv->n_kv_heads;
  a->n_q = n_q;
  a->S = S;
  a->G = G;
  a->cols = cols;
  a->pcols = G > 0 ? prefix_cols : 0;
  *bytes = paged_attention_workspace(*a, kv->dtype, kv->head_dim);
  if (*bytes == 0) return bad("the call's tables span too many key blocks");
  *bytes += 256;  // the workspace's parts start on 256-byte boundaries
  return ZSAA_OK;
}

zsaa_status select_sizes(int B, int W, int V, int K, size_t* stat, size_t* cand) {
  if (B < 1 || V < 1) return bad("B and V must be >= 1");
  if (W < 1 || W > kBeamMaxBeams || K < 1 || K > kBeamMaxKept)
    return refuse(ZSAA_ERR_INVALID_ARG, "W=%d or K=%d outside [1, 64]", W, K);
  if (V > kBeamMaxVocab) return bad("V must be at most 2^26");
  if (static_cast<long long>(W) * V < K) return bad("K exceeds the W*V continuations");
  const long long chunks = beam_chunks_most(V);
  if (static_cast<long long>(B) * W > kMostInt / 64 / chunks) return bad("B*W*V too large");
  *stat = (static_cast<size_t>(B) * W * chunks * sizeof(BeamChunk) + 255) & ~static_cast<size_t>(255);
  *cand = static_cast<size_t>(B) * W * chunks * K * sizeof(uint2);
  return ZSAA_OK;
}

}  // namespace

extern "C" {

zsaa_status zsaa_op_paged_append(const zsaa_pages* kv, const void* qkv, int64_t ld, int qkv_dtype, int T, int Hq,
                                 const int32_t* pos, float rope_theta, const int32_t* cu_rows, int S,
                                 const int32_t* table, int cols, const int32_t* lens, void* q_out,
                                 zsaa_stream stream) {
  ZTRY(check_pages(kv));
  ZTRY(check_pool(kv));
  if (qkv == nullptr || pos == nullptr || table == nullptr || lens == nullptr) return bad("null argument");
  if (!words(pos, cu_rows, table, lens)) return bad("int32 arrays must be 4-byte aligned");
  if (T < 1 || S < 1 || Hq < 1) return bad("T, S and Hq must be >= 1");
  if (cu_rows == nullptr && T != S) return bad("without cu_rows every sequence has one row: T must equal S");
  if (Hq % kv->n_kv_heads != 0) return bad("Hq must be a multiple of n_kv_heads");
  if (qkv_dtype != ZSAA_F32 && qkv_dtype != kv->dtype) return bad("qkv must be float32 or of the pool's dtype");
  if (!(rope_theta >= 1.f) || !std::isfinite(rope_theta)) return bad("rope_theta must be finite and >= 1");
  ZTRY(check_cols(cols, kv->page_size));
  const long long heads = static_cast<long long>(Hq) + 2LL * kv->n_kv_heads;
  if (heads > kMostInt / 1024) return bad("too many heads");
  const size_t e = element(qkv_dtype);
  if (ld < heads * kv->head_dim || ld > (1LL << 40)) return bad("ld is shorter than a row");
  if (!aligned(qkv, 16) || ld * e % 16 != 0 || !aligned(q_out, 16))
    return bad("qkv rows and q_out must be 16-byte aligned");
  const size_t q_bytes = static_cast<size_t>(T) * Hq * kv->head_dim * element(kv->dtype);
  if (q_out != nullptr && overlap(q_out, q_bytes, qkv, static_cast<size_t>(T) * ld * e))
    return bad("q_out overlaps qkv");
  int sms = 0;
  AppendArgs a{};
  ZTRY(device_sms(&sms));
  ZTRY(status_word(&a.status));
  a.k = kv->k, a.v = kv->v, a.qkv = qkv, a.q_out = q_out;
  a.pos = pos, a.cu_rows = cu_rows, a.table = table, a.lens = lens;
  a.ld = ld, a.T = T, a.S = S, a.cols = cols, a.Hq = Hq, a.Hkv = kv->n_kv_heads;
  a.n_pages = kv->n_pages, a.page_shift = page_shift(kv->page_size);
  return launched("zsaa_op_paged_append",
                  launch_paged_append(a, qkv_dtype, kv->dtype, kv->head_dim, rope_theta, sms,
                                      reinterpret_cast<cudaStream_t>(stream)));
}

zsaa_status zsaa_op_paged_attention_workspace(const zsaa_pages* kv, int S, int n_q, int Hq, int G, int cols,
                                              int prefix_cols, size_t* bytes) {
  if (bytes == nullptr) return bad("null bytes");
  *bytes = 0;
  PagedArgs a;
  return attention_sizes(kv, S, n_q, Hq, G, cols, prefix_cols, &a, bytes);
}

zsaa_status zsaa_op_paged_attention(const zsaa_pages* kv, const void* q, int S, int n_q, int Hq, const int32_t* table,
                                    int cols, const int32_t* lens, const int32_t* cu_seqs, int G,
                                    const int32_t* prefix_table, int prefix_cols, const int32_t* prefix_lens,
                                    void* out, float* lse, void* ws, size_t ws_bytes, zsaa_stream stream) {
  PagedArgs a;
  size_t need = 0;
  ZTRY(attention_sizes(kv, S, n_q, Hq, G, cols, prefix_cols, &a, &need));
  ZTRY(check_pool(kv));
  if (q == nullptr || table == nullptr || lens == nullptr || out == nullptr || ws == nullptr) return bad("null argument");
  if (G > 0 && (cu_seqs == nullptr || prefix_table == nullptr || prefix_lens == nullptr))
    return bad("groups need cu_seqs, prefix_table and prefix_lens");
  if (!words(table, lens, lse) || (G > 0 && !words(cu_seqs, prefix_table, prefix_lens)))
    return bad("int32 and float32 arrays must be 4-byte aligned");
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(ws, 16)) return bad("q, out and ws must be 16-byte aligned");
  if (ws_bytes < need) return refuse(ZSAA_ERR_INVALID_ARG, "ws_bytes %zu, needs %zu", ws_bytes, need);
  const size_t q_bytes = static_cast<size_t>(S) * n_q * Hq * kv->head_dim * element(kv->dtype);
  if (overlap(q, q_bytes, out, q_bytes)) return bad("out overlaps q");
  int sms = 0;
  ZTRY(device_sms(&sms));
  ZTRY(status_word(&a.status));
  a.k = kv->k, a.v = kv->v, a.q = q, a.out = out, a.lse = lse;
  a.table = table, a.lens = lens;
  if (G > 0) a.cu_seqs = cu_seqs, a.ptable = prefix_table, a.plens = prefix_lens;
  a.scale_log2 = 1.4426950408889634f / std::sqrt(static_cast<float>(kv->head_dim));
  void* at = reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(ws) + 255) & ~static_cast<uintptr_t>(255));
  return launched("zsaa_op_paged_attention", launch_paged_attention(a, kv->dtype, kv->head_dim, at, sms,
                                                                    reinterpret_cast<cudaStream_t>(stream)));
}

zsaa_status zsaa_op_beam_select_workspace(int B, int W, int V, int K, size_t* bytes) {
  if (bytes == nullptr) return bad("null bytes");
  *bytes = 0;
  size_t stat = 0, cand = 0;
  ZTRY(select_sizes(B, W, V, K, &stat, &cand));
  *bytes = stat + cand;
  return ZSAA_OK;
}

zsaa_status zsaa_op_beam_select(const float* logits, int64_t ld, int B, int W, int V, const float* scores,
                                const uint8_t* done, int eos, int K, float* scores_out, int32_t* parent,
                                int32_t* token, uint8_t* done_out, void* ws, size_t ws_bytes, zsaa_stream stream) {
  size_t stat = 0, cand = 0;
  ZTRY(select_sizes(B, W, V, K, &stat, &cand));
  if (logits == nullptr || scores_out == nullptr || parent == nullptr || token == nullptr || ws == nullptr)
    return bad("null argument");
  if (ld < V || ld > (1LL << 40)) return bad("ld is shorter than V");
  if (!words(logits, scores, scores_out, parent, token)) return bad("int32 and float32 arrays must be 4-byte aligned");
  if (eos < -1 || eos >= V) return bad("eos must be a token or -1");
  if (done != nullptr && eos < 0) return bad("done needs an eos token");
  if (!aligned(ws, 16)) return bad("ws must be 16-byte aligned");
  if (ws_bytes < stat + cand) return refuse(ZSAA_ERR_INVALID_ARG, "ws_bytes %zu, needs %zu", ws_bytes, stat + cand);
  const size_t in = static_cast<size_t>(B) * W, out = static_cast<size_t>(B) * K;
  if (scores != nullptr && overlap(scores, 4 * in, scores_out, 4 * out)) return bad("scores_out overlaps scores");
  if (done != nullptr && done_out != nullptr && overlap(done, in, done_out, out)) return bad("done_out overlaps done");
  int sms = 0;
  ZTRY(device_sms(&sms));
  return launched("zsaa_op_beam_select",
                  launch_beam_select(logits, ld, B, W, V, scores, done, eos, K, scores_out, parent, token, done_out,
                                     static_cast<BeamChunk*>(ws),
                                     reinterpret_cast<uint2*>(static_cast<char*>(ws) + stat), sms,
                                     reinterpret_cast<cudaStream_t>(stream)));
}

zsaa_status zsaa_op_beam_reorder(const zsaa_pages* layers, int n_layers, int B, int W, int K, const int32_t* parent,
                                 const int32_t* table, int32_t* table_out, int cols, const int32_t* lens,
                                 int32_t* lens_out, const int32_t* fresh, zsaa_stream stream) {
  if (layers == nullptr || parent == nullptr || table == nullptr || table_out == nullptr || lens == nullptr ||
      lens_out == nullptr || fresh == nullptr)
    return bad("null argument");
  if (!words(parent, table, table_out, lens, lens_out, fresh)) return bad("int32 arrays must be 4-byte aligned");
  if (n_layers < 1 || n_layers > kReorderMaxLayers) return refuse(ZSAA_ERR_INVALID_ARG, "n_layers=%d outside [1, 64]", n_layers);
  const void *k[kReorderMaxLayers], *v[kReorderMaxLayers];
  for (int l = 0; l < n_layers; ++l) {
    const zsaa_pages& p = layers[l];
    ZTRY(check_pages(&p));
    ZTRY(check_pool(&p));
    if (p.n_pages != layers[0].n_pages || p.page_size != layers[0].page_size || p.n_kv_heads != layers[0].n_kv_heads ||
        p.head_dim != layers[0].head_dim || p.dtype != layers[0].dtype)
      return bad("the layers' pools must have the same sizes and dtype");
    k[l] = p.k;
    v[l] = p.v;
  }
  if (B < 1) return bad("B must be >= 1");
  if (W < 1 || W > kBeamMaxBeams || K < 1 || K > kBeamMaxKept)
    return refuse(ZSAA_ERR_INVALID_ARG, "W=%d or K=%d outside [1, 64]", W, K);
  if (B > kMostInt / 64) return bad("too many sequences");
  const zsaa_pages& p = layers[0];
  ZTRY(check_cols(cols, p.page_size));
  const size_t in = 4 * static_cast<size_t>(B) * W, out = 4 * static_cast<size_t>(B) * K;
  if (overlap(table, in * cols, table_out, out * cols)) return bad("table_out overlaps table");
  if (overlap(lens, in, lens_out, out)) return bad("lens_out overlaps lens");
  int* status = nullptr;
  ZTRY(status_word(&status));
  return launched("zsaa_op_beam_reorder",
                  launch_beam_reorder(k, v, n_layers, p.n_pages, page_shift(p.page_size), p.n_kv_heads,
                                      static_cast<int>(p.head_dim * element(p.dtype)), B, W, K, parent, table,
                                      table_out, cols, lens, lens_out, fresh, status,
                                      reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
