// Declarations shared by the kernels on the evictable paged cache of the layers below the split: addressing, and one
// launcher per .cu file.
#pragma once
#include "earn_common.cuh"

namespace earn {

struct PagedSource {
  char *k, *v;                 // [n_pages, 16, Hkv, D]
  const int32_t* block_table;  // [B, pages_per_seq] or null (identity)
  const int32_t* seq_len;      // [B]
  int pages_per_seq, n_pages, max_len;
};
// page that holds rows 16 p .. of sequence b; `ok` tells whether the table names one (its number is clamped to the pool)
__device__ __forceinline__ int paged_page(const PagedSource& s, int b, int p, bool& ok) {
  const int64_t at = (int64_t)b * s.pages_per_seq + p;
  const int page = s.block_table ? s.block_table[at] : (int)at;
  ok = page >= 0 && page < s.n_pages;
  return min(max(page, 0), s.n_pages - 1);
}
__device__ __forceinline__ int paged_len(const PagedSource& s, int b) { return min(max(s.seq_len[b], 0), s.max_len); }

struct KeyWeightArgs {
  const void *q, *k;
  const float* lse;            // [Hq, total]
  float* weight;               // [Hkv, total]
  const int32_t* cu_seqlens;
  const int32_t* cu_seqlens_host;
  int batch, total, max_seqlen, n_obs, Hq, Hkv, D, dtype;
  float scale;
};
cudaError_t launch_key_weights_simt(const KeyWeightArgs& a, cudaStream_t st);
// tensor-core path (bf16, groups of at most 128 heads): one plan entry per key_weights_tc_rows() keys of a sequence
int key_weights_tc_rows();
bool key_weights_tc_supported(const KeyWeightArgs& a, int64_t plan_entries);
cudaError_t launch_key_weights_tc(const KeyWeightArgs& a, int plan_entries, void* plan, int32_t* status_word, cudaStream_t st);

struct EvictArgs {
  PagedSource cache;
  const void *k_packed, *v_packed;   // prompt form: packed [total, Hkv, D]; null: in place
  const int32_t* cu_seqlens;         // prompt form
  const float* weight;               // prompt form [Hkv, total], else [B, Hkv, cap]
  const int32_t* pos;                // in place: [B, Hkv, cap]
  float* weight_out;                 // [B, Hkv, cap] or null (prompt form)
  int32_t* pos_out;                  // [B, Hkv, cap]
  int32_t* moves;                    // in place: scratch [B * Hkv, 2, list] of (from, to) rows
  int32_t* n_moves;                  // in place: scratch [B * Hkv]
  int n_seq, total, max_rows, Hkv, row_bytes, budget, n_first, n_last, list;   // row_bytes: one head's row; max_rows: longest sequence
};
cudaError_t launch_evict(const EvictArgs& a, cudaStream_t st);

struct PagedDecodeArgs {
  const void *q, *k_new, *v_new;
  void* o;
  PagedSource cache;
  const float* weight;         // [B, Hkv, cap] or null (zeros)
  float* weight_out;           // or null
  const int32_t* new_pos;
  int32_t* pos;
  float* scores;               // [B, Hkv, g, score_ld] scaled log2-domain logits (only with weight_out)
  float* part_o;               // [B, Hkv, n_splits, g, D]
  float* part_lse;             // [B, Hkv, n_splits, g] (log2 domain)
  int n_seq, Hq, Hkv, D, dtype, g, cluster, chunk, n_splits, score_ld;
  float scale;
};
// How the key lists are cut.  cluster > 0: to the CTAs of a cluster, at most `chunk` rows each, in one launch without scratch
// (n_splits 0).  Otherwise n_splits chunks of `chunk` rows (a multiple of 16) and a second kernel that joins them.
struct PagedPlan {
  int cluster, chunk, n_splits;
};
constexpr int kPagedMaxChunk = 512;
PagedPlan plan_paged_decode(int n_seq, int n_kv_heads, int g, int max_len, int dtype);
cudaError_t launch_paged_decode(const PagedDecodeArgs& a, cudaStream_t st);

}  // namespace earn
