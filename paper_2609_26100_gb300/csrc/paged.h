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
};
size_t pa_partial_rows(int sms, int head_dim);
int pa_counters(int sms);
cudaError_t pa_prepare_all();
// *too_large: more work than one launch counts (nothing was launched).
cudaError_t launch_paged_attention(tss_paged* h, const PgAttnArgs& a, const PgBatch& batch, cudaStream_t s, bool* too_large);

}  // namespace tss
