// Host-side launchers of the paged-cache and beam-search kernels (internal; not part
// of the C ABI).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace zsaa {

// ---- paged caches (k_paged.cu): pools of pages [n_pages, Hkv, page, hd]
// Rotation frequencies of dims c, c + hd/2 as 64-bit fractions of a turn.
struct RopeTurns {
  unsigned long long f[64];
};
struct AppendArgs {
  void *k, *v;
  const void* qkv;
  void* q_out;  // or null
  const int32_t *pos, *cu_rows, *table, *lens;  // cu_rows null: one row per sequence
  long long ld;
  int T, S, cols, Hq, Hkv, n_pages, page_shift;
  int* status;
};
cudaError_t launch_paged_append(const AppendArgs& a, int in_dtype, int dtype, int hd, float theta, int sms,
                                cudaStream_t s);

struct PagedArgs {
  const void *k, *v, *q;
  void* out;
  float* lse;  // or null
  int n_pages, page_shift, Hkv, per, n_q, S, G, cols, pcols;
  const int32_t *table, *lens, *cu_seqs, *ptable, *plens;
  float scale_log2;
  int* status;
};
// One attention launch's entries and its part of the workspace (paged.cuh).
struct PagedWork {
  int e0, e1;      // entries [e0, e1) of the groups' prefixes, then the sequences
  int min_units;   // a CTA's stretch is at least this long
  int lead;        // units of an item before its blocks
  int mt_shift, bn_shift;  // rows of a tile, keys of a block: powers of two
  int* head;       // [1 + entries]
  float* o;        // [slots][rows of a tile][hd]
  float* lse2;     // [slots][rows of a tile]
};
// A kernel's tiles, the CTAs it is launched with, the least units a CTA takes, and the blocks
// that an item's start and end take the time of.
struct PagedTiles {
  int mt, bn, ctas, min_units, lead;
};
// tiles of 16 rows (k_paged_mma.cu)
PagedTiles paged_mma_tiles(int dtype, int hd, int sms);
cudaError_t launch_paged_mma(const PagedArgs& a, const PagedWork& w, int dtype, int hd, int ctas, cudaStream_t s);
// all of a sequence and KV head's keys in one CTA; prefixes: the launch that has left the
// prefixes' partial results (bf16), or null
cudaError_t launch_paged_direct(const PagedArgs& a, const PagedWork* prefixes, int dtype, int hd, cudaStream_t s);
// bf16, tiles of 128 rows (k_paged_tc.cu)
PagedTiles paged_tc_tiles(int sms);
cudaError_t launch_paged_tc(const PagedArgs& a, const PagedWork& w, int hd, int ctas, cudaStream_t s);
// Bytes of workspace that a call of these sizes needs (0: sizes beyond its index range).
size_t paged_attention_workspace(const PagedArgs& a, int dtype, int hd);
cudaError_t launch_paged_attention(const PagedArgs& a, int dtype, int hd, void* ws, int sms, cudaStream_t s);

// ---- beam search (k_beam.cu)
constexpr int kBeamMaxBeams = 64, kBeamMaxKept = 64, kBeamMaxVocab = 1 << 26;
constexpr int kReorderMaxLayers = 64;
struct BeamChunk {
  unsigned long long sum;  // sum of exp(x - top) in units of 2^-36
  float top;               // the maximum
  int bad;                 // a NaN or +inf among the logits
};
// Stretches that a beam's logits are scanned in, at most, on any device.
int beam_chunks_most(int V);
cudaError_t launch_beam_select(const float* logits, long long ld, int B, int W, int V, const float* scores,
                               const uint8_t* done, int eos, int K, float* scores_out, int32_t* parent,
                               int32_t* token, uint8_t* done_out, BeamChunk* stat, uint2* cand, int sms,
                               cudaStream_t s);
cudaError_t launch_beam_reorder(const void* const* k, const void* const* v, int n_layers, int n_pages, int page_shift,
                                int Hkv, int entry_bytes, int B, int W, int K, const int32_t* parent,
                                const int32_t* table, int32_t* table_out, int cols, const int32_t* lens,
                                int32_t* lens_out, const int32_t* fresh, int* status, cudaStream_t s);

// ---- status word of the calls without a model (zsaa_api.cu): the current device's, or null
int* shared_status_word();

}  // namespace zsaa
