// C ABI of the paged-cache, beam-search and draft-verification calls: argument checks and launches.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>

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

// Arrays that a call writes lie over none that it reads, and over no other that it writes.
struct Array {
  const void* p;  // or null
  size_t bytes;
};
bool apart(std::initializer_list<Array> written, std::initializer_list<Array> read) {
  for (const Array* w = written.begin(); w != written.end(); ++w) {
    if (w->p == nullptr) continue;
    for (const Array* o = w + 1; o != written.end(); ++o)
      if (o->p != nullptr && overlap(w->p, w->bytes, o->p, o->bytes)) return false;
    for (const Array& r : read)
      if (r.p != nullptr && overlap(w->p, w->bytes, r.p, r.bytes)) return false;
  }
  return true;
}
// with any of n rows of `width` bytes, `stride` bytes apart (what lies between them is no part of them)
bool overlap_rows(const void* a, size_t an, const void* rows, size_t n, size_t stride, size_t width) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), r = reinterpret_cast<uintptr_t>(rows);
  if (x <= r) return r - x < an;
  const uintptr_t row = (x - r) / stride, at = (x - r) % stride;  // the last row that starts at or before x
  return row < n && (at < width || (row + 1 < n && stride - at < an));
}

constexpr long long kMostInt = 0x7fffffff;
constexpr int kMostPages = 1 << 30;

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

// the layers' pools of a call that moves entries in all of them
zsaa_status check_layers(const zsaa_pages* layers, int n_layers, PoolList* pools) {
  if (layers == nullptr) return bad("null layers");
  if (n_layers < 1 || n_layers > kReorderMaxLayers) return refuse(ZSAA_ERR_INVALID_ARG, "n_layers=%d outside [1, 64]", n_layers);
  for (int l = 0; l < n_layers; ++l) {
    const zsaa_pages& p = layers[l];
    ZTRY(check_pages(&p));
    ZTRY(check_pool(&p));
    if (p.n_pages != layers[0].n_pages || p.page_size != layers[0].page_size || p.n_kv_heads != layers[0].n_kv_heads ||
        p.head_dim != layers[0].head_dim || p.dtype != layers[0].dtype)
      return bad("the layers' pools must have the same sizes and dtype");
    pools->p[2 * l] = p.k;
    pools->p[2 * l + 1] = p.v;
  }
  pools->n = 2 * n_layers;
  return ZSAA_OK;
}

// The pools, each once: layers may share a cache, keys and values a pool, and entries that move in
// place are moved by one CTA's reads and writes alone.
PoolList each_once(const PoolList& given) {
  PoolList out{};
  for (int i = 0; i < given.n; ++i) {
    bool again = false;
    for (int j = 0; j < out.n; ++j) again |= out.p[j] == given.p[i];
    if (!again) out.p[out.n++] = given.p[i];
  }
  return out;
}

// (a grid's third dimension, 4 CTAs to a head; a page's vectors in 31 bits)
zsaa_status check_heads(int n) { return n <= 16383 ? ZSAA_OK : bad("more than 16383 KV heads"); }

// rows of a table whose pages a call takes
zsaa_status check_taking(int rows, int cols, int page) {
  if (rows < 1) return bad("a table needs 1 or more rows");
  if (rows > kPagesMaxRows) return refuse(ZSAA_ERR_UNSUPPORTED, "%d rows of pages, the most are %d", rows, kPagesMaxRows);
  ZTRY(check_cols(cols, page));
  if (static_cast<long long>(rows) * cols > kMostInt) return bad("a table must have fewer than 2^31 entries");
  return ZSAA_OK;
}

// offsets of a verification's parts in its workspace: stretches, groups, decisions
zsaa_status verify_sizes(int S, int n, int V, size_t* groups, size_t* state, size_t* bytes) {
  if (S < 1 || V < 1) return bad("S and V must be >= 1");
  if (n < 0 || n > kVerifyMaxDrafts) return refuse(ZSAA_ERR_UNSUPPORTED, "n=%d drafts outside [0, %d]", n, kVerifyMaxDrafts);
  if (V > kVerifyMaxVocab) return bad("V must be at most 2^26");
  const long long items = static_cast<long long>(2 * n + 1) * verify_chunks(V);
  if (S > kMostInt / 16 / items) return bad("S*n*V too large");
  *groups = (static_cast<size_t>(S) * items * sizeof(VerifyChunk) + 31) & ~static_cast<size_t>(31);
  *state = *groups + static_cast<size_t>(S) * verify_groups_most(V) * sizeof(VerifyGroup);
  *bytes = *state + static_cast<size_t>(S) * sizeof(VerifyState);
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
  PoolList pools{};
  ZTRY(check_layers(layers, n_layers, &pools));
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
                  launch_beam_reorder(pools, p.n_pages, page_shift(p.page_size), p.n_kv_heads,
                                      static_cast<int>(p.head_dim * element(p.dtype)), B, W, K, parent, table,
                                      table_out, cols, lens, lens_out, fresh, status,
                                      reinterpret_cast<cudaStream_t>(stream)));
}

zsaa_status zsaa_op_paged_resize(int32_t* refs, int n_pages, int page_size, int S, int32_t* table, int cols,
                                 const int32_t* lens, const int32_t* want, int32_t* lens_out, int32_t* n_free,
                                 zsaa_stream stream) {
  if (refs == nullptr || table == nullptr || lens == nullptr || want == nullptr || lens_out == nullptr)
    return bad("null argument");
  if (!words(refs, table, lens, want, lens_out, n_free)) return bad("int32 arrays must be 4-byte aligned");
  if (n_pages < 1 || n_pages > kMostPages) return bad("n_pages must be in [1, 2^30]");
  if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0)
    return refuse(ZSAA_ERR_UNSUPPORTED, "page_size %d is not 16, 32, 64, 128 or 256", page_size);
  ZTRY(check_taking(S, cols, page_size));
  const size_t row = 4 * static_cast<size_t>(S);
  if (!apart({{refs, 4 * static_cast<size_t>(n_pages)}, {table, row * cols}, {lens_out, row}, {n_free, 4}}, {{lens, row}, {want, row}}))
    return bad("refs, table, lens_out or n_free overlaps another array");
  PagesArgs a{};
  ZTRY(status_word(&a.status));
  a.refs = refs, a.table = a.table_out = table, a.lens = lens, a.want = want, a.lens_out = lens_out, a.n_free = n_free;
  a.rows = S, a.cols = cols, a.n_pages = n_pages, a.page_shift = page_shift(page_size);
  return launched("zsaa_op_paged_resize", launch_paged_resize(a, reinterpret_cast<cudaStream_t>(stream)));
}

zsaa_status zsaa_op_paged_fork(const zsaa_pages* layers, int n_layers, int32_t* refs, int S, const int32_t* table, int cols,
                               const int32_t* lens, int N, const int32_t* parent, const int32_t* at, int32_t* table_out,
                               int32_t* lens_out, int32_t* n_free, zsaa_stream stream) {
  PoolList pools{};
  ZTRY(check_layers(layers, n_layers, &pools));
  if (refs == nullptr || table == nullptr || lens == nullptr || parent == nullptr || table_out == nullptr ||
      lens_out == nullptr)
    return bad("null argument");
  if (!words(refs, table, lens, parent, at, table_out, lens_out, n_free)) return bad("int32 arrays must be 4-byte aligned");
  const zsaa_pages& p = layers[0];
  if (S < 1) return bad("S must be >= 1");
  ZTRY(check_heads(p.n_kv_heads));
  ZTRY(check_taking(N, cols, p.page_size));
  if (static_cast<long long>(S) * cols > kMostInt) return bad("a table must have fewer than 2^31 entries");
  const size_t in = 4 * static_cast<size_t>(S), out = 4 * static_cast<size_t>(N);
  if (!apart({{refs, 4 * static_cast<size_t>(p.n_pages)}, {table_out, out * cols}, {lens_out, out}, {n_free, 4}},
             {{table, in * cols}, {lens, in}, {parent, out}, {at, out}}))
    return bad("refs, table_out, lens_out or n_free overlaps another array");
  PagesArgs a{};
  ZTRY(status_word(&a.status));
  a.refs = refs, a.table = table, a.table_out = table_out, a.lens = lens, a.parent = parent, a.at = at;
  a.lens_out = lens_out, a.n_free = n_free;
  a.rows = N, a.cols = cols, a.n_pages = p.n_pages, a.page_shift = page_shift(p.page_size), a.parents = S;
  return launched("zsaa_op_paged_fork",
                  launch_paged_fork(a, pools, p.n_kv_heads, static_cast<int>(p.head_dim * element(p.dtype) / 16),
                                    reinterpret_cast<cudaStream_t>(stream)));
}

zsaa_status zsaa_op_paged_compact(const zsaa_pages* layers, int n_layers, const int32_t* refs, int S, const int32_t* table,
                                  int cols, const int32_t* lens, const int32_t* start, const int32_t* keep, int keep_cols,
                                  const int32_t* n_keep, const int32_t* table_out, int out_cols, int32_t* lens_out,
                                  zsaa_stream stream) {
  PoolList pools{};
  ZTRY(check_layers(layers, n_layers, &pools));
  if (table == nullptr || lens == nullptr || keep == nullptr || n_keep == nullptr || table_out == nullptr ||
      lens_out == nullptr)
    return bad("null argument");
  if (!words(refs, table, lens, start, keep, n_keep, table_out, lens_out)) return bad("int32 arrays must be 4-byte aligned");
  const zsaa_pages& p = layers[0];
  if (S < 1 || keep_cols < 1) return bad("S and keep_cols must be >= 1");
  ZTRY(check_heads(p.n_kv_heads));
  ZTRY(check_cols(cols, p.page_size));
  ZTRY(check_cols(out_cols, p.page_size));
  const size_t row = 4 * static_cast<size_t>(S);
  if (!apart({{lens_out, row}}, {{table, row * cols}, {lens, row}, {start, row}, {keep, row * keep_cols}, {n_keep, row},
                                 {table_out, row * out_cols}, {refs, 4 * static_cast<size_t>(p.n_pages)}}))
    return bad("lens_out overlaps another array");
  // a sequence's row of one must not be another's, or another column of its own, of the other
  const bool in_place = table_out == table && (out_cols == cols || S == 1);
  if (!in_place && overlap(table, row * cols, table_out, row * out_cols))
    return bad("table_out overlaps table and is not the same array of the same width");
  int sms = 0;
  ZTRY(device_sms(&sms));
  CompactArgs a{};
  ZTRY(status_word(&a.status));
  a.table = table, a.lens = lens, a.start = start, a.keep = keep, a.n_keep = n_keep, a.table_out = table_out, a.refs = refs;
  a.lens_out = lens_out;
  a.S = S, a.cols = cols, a.out_cols = out_cols, a.keep_cols = keep_cols, a.n_pages = p.n_pages;
  a.page_shift = page_shift(p.page_size), a.Hkv = p.n_kv_heads;
  a.row_vecs = static_cast<int>(p.head_dim * element(p.dtype) / 16);
  return launched("zsaa_op_paged_compact", launch_paged_compact(a, each_once(pools), sms, reinterpret_cast<cudaStream_t>(stream)));
}

zsaa_status zsaa_op_draft_verify_workspace(int S, int n, int V, size_t* bytes) {
  if (bytes == nullptr) return bad("null bytes");
  *bytes = 0;
  size_t groups = 0, state = 0;
  return verify_sizes(S, n, V, &groups, &state, bytes);
}

zsaa_status zsaa_op_draft_verify(const void* target, int64_t ld, const void* draft, int64_t draft_ld, int dtype, int S, int n,
                                 int V, const int32_t* drafts, const float* temperature, const float* uniform,
                                 int32_t* accepted, int32_t* tokens, float* logp, const int32_t* lens, int32_t* lens_out,
                                 void* ws, size_t ws_bytes, zsaa_stream stream) {
  size_t groups = 0, state = 0, need = 0;
  ZTRY(verify_sizes(S, n, V, &groups, &state, &need));
  if (dtype != ZSAA_F32 && dtype != ZSAA_BF16) return bad("bad dtype");
  if (n == 0) drafts = nullptr, draft = nullptr;
  if (target == nullptr || (n > 0 && drafts == nullptr) || uniform == nullptr || accepted == nullptr || tokens == nullptr ||
      ws == nullptr)
    return bad("null argument");
  if ((lens == nullptr) != (lens_out == nullptr)) return bad("lens and lens_out: both or neither");
  if (ld < V || ld > (1LL << 40)) return bad("ld is shorter than V");
  if (draft != nullptr && (draft_ld < V || draft_ld > (1LL << 40))) return bad("draft_ld is shorter than V");
  if (!aligned(target, element(dtype)) || !aligned(draft, element(dtype))) return bad("logits must be aligned to their type");
  if (!words(drafts, temperature, uniform, accepted, tokens, logp, lens, lens_out))
    return bad("int32 and float32 arrays must be 4-byte aligned");
  if (!aligned(ws, 16)) return bad("ws must be 16-byte aligned");
  if (ws_bytes < need) return refuse(ZSAA_ERR_INVALID_ARG, "ws_bytes %zu, needs %zu", ws_bytes, need);
  const size_t row = 4 * static_cast<size_t>(S);
  // CTAs of a sequence read what others of it write, so outputs and the workspace lie over nothing else (but
  // lens_out may be lens)
  const size_t e = element(dtype), drafted = draft != nullptr ? static_cast<size_t>(S) * n : 0, each = row * (n + 1);
  if (!apart({{accepted, row}, {tokens, each}, {logp, each}, {lens_out, row}, {ws, need}},
             {{lens != lens_out ? lens : nullptr, row}, {drafts, row * n}, {temperature, row}, {uniform, each}}))
    return bad("an output or the workspace overlaps another array");
  for (const Array& o : {Array{accepted, row}, {tokens, each}, {logp, each}, {lens_out, row}, {ws, need}}) {
    if (o.p == nullptr) continue;
    if (overlap_rows(o.p, o.bytes, target, static_cast<size_t>(S) * (n + 1), ld * e, V * e) ||
        (drafted > 0 && overlap_rows(o.p, o.bytes, draft, drafted, draft_ld * e, V * e)))
      return bad("an output or the workspace overlaps the logits");
  }
  int sms = 0;
  ZTRY(device_sms(&sms));
  VerifyArgs a{};
  a.target = target, a.draft = draft, a.ld = ld, a.draft_ld = draft_ld;
  a.S = S, a.n = n, a.V = V, a.chunks = verify_chunks(V), a.rows = n + 1 + (draft != nullptr ? n : 0);
  a.drafts = drafts, a.lens = lens, a.temperature = temperature, a.uniform = uniform;
  a.accepted = accepted, a.tokens = tokens, a.lens_out = lens_out, a.logp = logp;
  a.stat = static_cast<VerifyChunk*>(ws);
  a.groups = reinterpret_cast<VerifyGroup*>(static_cast<char*>(ws) + groups);
  a.state = reinterpret_cast<VerifyState*>(static_cast<char*>(ws) + state);
  return launched("zsaa_op_draft_verify", launch_draft_verify(a, dtype, sms, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
