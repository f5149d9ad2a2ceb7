// The 4-bit paged cache's workspace and the attention's launch interface.
#pragma once

#include "ops.cuh"

// (opaque in tss.h)
struct tss_paged {
  int hq, hk, d, dev, sms;
  int* status;      // device
  float* part_o;    // device: partial results of items that several CTAs share
  float2* part_ml;
  int* counters;    // device [pa_counters], zero between launches
  int inject;       // attention launches still to be made to run out of time (tests)
  int share_rows;   // rows that a shared attention may have
  float* share_o;   // device [share_rows][hq][d]: results over the shared keys, unnormalised
  float2* share_ml; // device [share_rows][hq]: their references and sums
  float* own_o;     // part_o, part_ml and counters of the pass over own keys, which overlaps the one over shared keys
  float2* own_ml;
  int* own_counters;
};

namespace tss {

struct PgAttnArgs {
  int hq, hk, d, n_pages, max_pages;
  const uint8_t* pool;      // the layer's pages
  const int* table;
  const void* q;
  void* out;
  float* lse;
  long long qs, os;
  float scale_log2;         // scale * log2(e)
  int window, sinks, is_half;
  const unsigned long long* mask;
  const int* positions;
  int* status;
  // attention of sequences that share keys, in two passes
  int own;                  // 0: over the shared keys, results to share_*; 1: over a request's own, joined with those
  float* share_o;
  float2* share_ml;
};
// Checks what every call on the cache has in common and copies the batch.  *rows: rows in all.
tss_status take_batch(const tss_paged* h, const tss_paged_cache* c, int layer, const tss_paged_batch* b, PgBatch* out, long long* rows);
cudaError_t append_rope_prepare();
size_t pa_partial_rows(int sms, int head_dim);
int pa_counters(int sms);
cudaError_t pa_prepare_all();
// *too_large: more work than one launch counts (nothing was launched).
cudaError_t launch_paged_attention(tss_paged* h, const PgAttnArgs& a, const PgBatch& batch, cudaStream_t s, bool* too_large);
// Groups of requests, one after the other, whose sequences have the same pages for the first `shared` tokens (a multiple of 64, at
// most the requests' first tokens).
struct PgGroups {
  int n;
  int reqs[kPgMaxReq], shared[kPgMaxReq];
};
cudaError_t launch_paged_attention_shared(tss_paged* h, const PgAttnArgs& a, const PgBatch& batch, const PgGroups& groups, cudaStream_t s,
                                          bool* too_large);

}  // namespace tss
