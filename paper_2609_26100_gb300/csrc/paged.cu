// The paged 4-bit KV cache: its workspace, appending (quantising) tokens and reading them back.
//
// Quantisation, per token and 64 dims:  z = fp16(min), s = fp16((max - z) / 15), c = rint((x - z) / s) (paged_quant.cuh).
//
// Bound: appending prompts, instruction issue (69 % of the slots, 17 instructions a value): 7171 rows of 40 heads of
// 128, bf16, 50 us, 3.8 TB/s of rows read and codes written.  Reading them back, HBM: 36 us, 5.2 TB/s.  A step's 16 rows:
// 4.4 us, launch and latency.
#include "paged_quant.cuh"

namespace tss {
namespace {

template <typename T, int D>
__global__ void __launch_bounds__(kPqThreads) append_kernel(const __grid_constant__ PqParams p) {
  const int lane = threadIdx.x & 31;
  griddep_wait();
  griddep_launch();
  PqUnit u;
  if (!pq_unit(p, pq_warp(), lane, &u)) return;
  const long long stride = u.side ? p.vs : p.ks;
  quantise_run<T, D>(p, u, static_cast<const T*>(u.side ? p.v : p.k) + u.row * stride + u.head * D, stride, lane);
}

template <typename T, int D>
__global__ void __launch_bounds__(kPqThreads) read_kernel(const __grid_constant__ PqParams p) {
  using B = PgBlock<D>;
  using L = PqLane<D>;
  const int lane = threadIdx.x & 31;
  griddep_wait();
  griddep_launch();
  PqUnit u;
  if (!pq_unit(p, pq_warp(), lane, &u)) return;
  pq_resolve(p, B::kBytes, lane, &u);
  T* dst = static_cast<T*>(u.side ? p.vo : p.ko);
  if (!dst) return;
  const L at(lane);
  const long long stride = u.side ? p.vs : p.ks;
  dst += u.row * stride + u.head * D + at.d0;
  const __half2* params = reinterpret_cast<const __half2*>(u.block + (u.side ? B::kVParams : B::kKParams)) + u.tok0 * B::kGroups + at.d0 / kPgGroup;
  const uint8_t* krow = u.block + B::kK + u.tok0 * (D / 2) + at.k_at;
  // V: 16 bits (the lane's token parity) of the words of its dims, [t][pair of dims]
  uint32_t words[L::kT][4];
  if (u.side && u.block) {
#pragma unroll
    for (int tl = 0; tl < L::kT; ++tl)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const uint4 v = reinterpret_cast<const uint4*>(u.block + B::kV)[(u.tok0 / 32 * (D / 4) + at.d0 / 4 + q) * 4 + at.t(tl)];
        const uint32_t sel = at.i ? 0x7632 : 0x5410;
        words[tl][2 * q] = __byte_perm(v.x, v.y, sel);
        words[tl][2 * q + 1] = __byte_perm(v.z, v.w, sel);
      }
  }
  // all of the run's loads first, then its tokens
  constexpr int kSteps = 32 / L::kTokens;
  uint32_t w[kSteps];
  __half2 sz[kSteps];
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const int tok = j * L::kTokens + at.sub;
    w[j] = 0;
    sz[j] = __half2half2(__ushort_as_half(0));
    if (tok >= u.lo && tok < u.hi && u.block) {  // (no such page: zeros)
      sz[j] = params[tok * B::kGroups];
      if (!u.side) w[j] = *reinterpret_cast<const uint32_t*>(krow + tok * (D / 2));
    }
  }
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const int tok = j * L::kTokens + at.sub;
    if (tok < u.lo || tok >= u.hi) continue;
    const float2 f = __half22float2(sz[j]);
    const f2_t s2 = f2_pack(f.x, f.x), z2 = f2_pack(f.y, f.y), less = f2_pack(-8388608.f, -8388608.f);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      // a code as a float: the low bits of 2^23 + c (the conversion instruction has an eighth of the rate)
      uint32_t c[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t m = u.side && u.block ? words[j % L::kT][e / 2] >> (16 * i + 4 * (tok / 8)) : w[j] >> (4 * (e + i));
        c[i] = (m & 15u) | 0x4b000000u;
      }
      const float2 y = f2_unpack(f2_fma(f2_add(f2_pack(__uint_as_float(c[0]), __uint_as_float(c[1])), less), s2, z2));
      x[e] = y.x;
      x[e + 1] = y.y;
    }
    store_vec<T, 8>(dst + (tok - u.lo) * stride, x);
  }
}

template <int D>
cudaError_t pq_launch(const PqParams& p, bool append, int dtype, unsigned grid, cudaStream_t s) {
  cudaError_t e;
#define TSS_PQ(T)                                      \
  if (append)                                          \
    e = launch_k(append_kernel<T, D>, dim3(grid), dim3(kPqThreads), 0, s, true, p); \
  else                                                 \
    e = launch_k(read_kernel<T, D>, dim3(grid), dim3(kPqThreads), 0, s, true, p)
  if (dtype == TSS_DTYPE_BF16) {
    TSS_PQ(__nv_bfloat16);
  } else if (dtype == TSS_DTYPE_F16) {
    TSS_PQ(__half);
  } else {
    TSS_PQ(float);
  }
#undef TSS_PQ
  return e;
}

}  // namespace

// Checks what every call on the cache has in common and copies the batch.  *rows: rows in all.
tss_status take_batch(const tss_paged* h, const tss_paged_cache* c, int layer, const tss_paged_batch* b, PgBatch* out, long long* rows) {
  if (!h || !c || !b) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  const tss_status on = still_on(h->dev);
  if (on != TSS_OK) return on;
  if (!c->layer || c->n_layers < 1 || layer < 0 || layer >= c->n_layers)
    return refuse(TSS_ERR_INVALID_ARG, "layer must be in [0, n_layers)");
  if (!c->layer[layer] || !aligned16(c->layer[layer])) return refuse(TSS_ERR_INVALID_ARG, "the layer's pages must be 16-byte aligned device memory");
  if (static_cast<long long>(c->n_pages) * h->hk >= 1 << 30) return refuse(TSS_ERR_INVALID_ARG, "n_pages * n_kv_heads must be below 2^30");
  if (!c->table || c->n_pages < 1 || c->n_seqs < 1 || c->max_pages < 1 || c->max_pages > (1 << 24))
    return refuse(TSS_ERR_INVALID_ARG, "the cache needs a table, n_pages and n_seqs >= 1 and max_pages in [1, 2^24]");
  if (b->n_req < 1 || b->n_req > kPgMaxReq) return refuse(TSS_ERR_INVALID_ARG, "n_req must be in [1, 64]");
  if (!b->seq || !b->first || !b->n_tokens) return refuse(TSS_ERR_INVALID_ARG, "the batch needs seq, first and n_tokens");
  long long at = 0;
  out->n_req = b->n_req;
  for (int i = 0; i < b->n_req; ++i) {
    if (b->seq[i] < 0 || b->seq[i] >= c->n_seqs) return refuse(TSS_ERR_INVALID_ARG, "seq must be in [0, n_seqs)");
    if (b->first[i] < 0 || b->n_tokens[i] < 0) return refuse(TSS_ERR_INVALID_ARG, "first and n_tokens must be >= 0");
    if (static_cast<long long>(b->first[i]) + b->n_tokens[i] > static_cast<long long>(c->max_pages) * kPgTokens)
      return refuse(TSS_ERR_KV_CAPACITY, "first + n_tokens exceeds 64 * max_pages");
    out->r[i] = PgReq{b->seq[i], b->first[i], b->n_tokens[i], static_cast<int>(at)};
    at += b->n_tokens[i];
    if (at > 0x7fffffffLL) return refuse(TSS_ERR_INVALID_ARG, "more than 2^31 - 1 rows");
  }
  *rows = at;
  return TSS_OK;
}

bool pq_once(const PgBatch& b) {
  for (int i = 0; i < b.n_req; ++i)
    for (int j = 0; j < i; ++j)
      if (b.r[i].seq == b.r[j].seq) return false;
  return true;
}

tss_status pq_take(const tss_paged* h, const tss_paged_cache* cache, int layer, const tss_paged_batch* batch, PqParams* p, long long* rows) {
  const tss_status st = take_batch(h, cache, layer, batch, &p->batch, rows);
  if (st != TSS_OK) return st;
  long long total = 0;
  for (int i = 0; i < p->batch.n_req; ++i) {
    const PgReq& r = p->batch.r[i];
    p->off[i] = static_cast<int>(total);
    if (r.n) total += (r.first + r.n - 1) / 32 - r.first / 32 + 1;
  }
  p->total = static_cast<int>(total);
  p->hk = h->hk;
  p->n_pages = cache->n_pages;
  p->max_pages = cache->max_pages;
  p->pool = static_cast<uint8_t*>(cache->layer[layer]);
  p->table = cache->table;
  p->status = h->status;
  return TSS_OK;
}

namespace {

tss_status quant_call(tss_paged* h, const tss_paged_cache* cache, int layer, const tss_paged_batch* batch, const void* k, const void* v,
                      void* ko, void* vo, int64_t ks, int64_t vs, int dtype, bool append, void* stream) {
  PqParams p{};
  long long rows = 0;
  const tss_status st = pq_take(h, cache, layer, batch, &p, &rows);
  if (st != TSS_OK) return st;
  if (!known_dtype(dtype)) return refuse(TSS_ERR_INVALID_ARG, "unknown dtype");
  if (append && !pq_once(p.batch)) return refuse(TSS_ERR_INVALID_ARG, "a sequence appears twice");
  if (rows == 0) return TSS_OK;
  const int64_t width = static_cast<int64_t>(h->hk) * h->d;
  const void* ps[2] = {append ? k : ko, append ? v : vo};
  const int64_t strides[2] = {ks, vs};
  if (append ? (!ps[0] || !ps[1]) : (!ps[0] && !ps[1])) return refuse(TSS_ERR_INVALID_ARG, "k or v is NULL");
  for (int i = 0; i < 2; ++i)
    if (ps[i] && (!aligned16(ps[i]) || !good_stride(strides[i], width, dtype)))
      return refuse(TSS_ERR_INVALID_ARG, "k and v must be 16-byte aligned, their row strides hold the heads and be multiples of 16 bytes");
  p.k = k;
  p.v = v;
  p.ko = ko;
  p.vo = vo;
  p.ks = ks;
  p.vs = vs;
  const long long warps = static_cast<long long>(p.total) * 2 * h->hk, per = kPqThreads / 32;
  if ((warps + per - 1) / per > 0x7fffffffLL) return refuse(TSS_ERR_INVALID_ARG, "too many rows for one launch");
  const unsigned grid = static_cast<unsigned>((warps + per - 1) / per);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = h->d == 64 ? pq_launch<64>(p, append, dtype, grid, s) : pq_launch<128>(p, append, dtype, grid, s);
  return e == cudaSuccess ? TSS_OK : refuse_cuda(e, "launch");
}

}  // namespace
}  // namespace tss

using namespace tss;

extern "C" size_t tss_paged_page_bytes(int n_kv_heads, int head_dim) {
  if (n_kv_heads < 1 || n_kv_heads > 1024) return 0;
  return pg_block_bytes(head_dim) * static_cast<size_t>(n_kv_heads);
}

extern "C" tss_status tss_paged_create(int n_q_heads, int n_kv_heads, int head_dim, tss_paged** out) {
  return tss_paged_create_shared(n_q_heads, n_kv_heads, head_dim, 0, out);
}

extern "C" tss_status tss_paged_create_shared(int n_q_heads, int n_kv_heads, int head_dim, int shared_rows, tss_paged** out) {
  if (!out) return refuse(TSS_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (head_dim != 64 && head_dim != 128) return refuse(TSS_ERR_INVALID_ARG, "head_dim must be 64 or 128");
  if (n_kv_heads < 1 || n_kv_heads > 1024) return refuse(TSS_ERR_INVALID_ARG, "n_kv_heads must be in [1, 1024]");
  if (n_q_heads < 1 || n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > 64)
    return refuse(TSS_ERR_INVALID_ARG, "n_q_heads must be a multiple of n_kv_heads, at most 64 times it");
  if (shared_rows < 0 || shared_rows > kPgMaxReq * kPgMaxRows) return refuse(TSS_ERR_INVALID_ARG, "shared_rows must be in [0, 8192]");
  int dev = 0, sms = 0;
  const tss_status st = this_device(&dev, &sms);
  if (st != TSS_OK) return st;
  tss_paged* h = new (std::nothrow) tss_paged{};
  if (!h) return refuse(TSS_ERR_OUT_OF_MEMORY, "no host memory");
  h->hq = n_q_heads;
  h->hk = n_kv_heads;
  h->d = head_dim;
  h->dev = dev;
  h->sms = sms;
  const size_t rows = pa_partial_rows(sms, head_dim);
  cudaError_t e = pa_prepare_all();
  if (e == cudaSuccess) e = append_rope_prepare();
  if (e == cudaSuccess) e = cudaMalloc(&h->status, 256);
  if (e == cudaSuccess) e = zero_now(h->status, 256);
  if (e == cudaSuccess) e = cudaMalloc(&h->part_o, rows * head_dim * sizeof(float));
  if (e == cudaSuccess) e = cudaMalloc(&h->part_ml, rows * sizeof(float2));
  if (e == cudaSuccess) e = cudaMalloc(&h->counters, pa_counters(sms) * sizeof(int));
  if (e == cudaSuccess) e = zero_now(h->counters, pa_counters(sms) * sizeof(int));
  const size_t share = static_cast<size_t>(shared_rows) * n_q_heads;
  h->share_rows = shared_rows;
  if (e == cudaSuccess && share) e = cudaMalloc(&h->share_o, share * head_dim * sizeof(float));
  if (e == cudaSuccess && share) e = cudaMalloc(&h->share_ml, share * sizeof(float2));
  if (e == cudaSuccess && share) e = cudaMalloc(&h->own_o, rows * head_dim * sizeof(float));
  if (e == cudaSuccess && share) e = cudaMalloc(&h->own_ml, rows * sizeof(float2));
  if (e == cudaSuccess && share) e = cudaMalloc(&h->own_counters, pa_counters(sms) * sizeof(int));
  if (e == cudaSuccess && share) e = zero_now(h->own_counters, pa_counters(sms) * sizeof(int));
  if (e != cudaSuccess) {
    tss_paged_destroy(h);
    const tss_status r = refuse_cuda(e, "workspace");
    return e == cudaErrorMemoryAllocation ? TSS_ERR_OUT_OF_MEMORY : r;
  }
  *out = h;
  return TSS_OK;
}

extern "C" void tss_paged_destroy(tss_paged* h) {
  if (!h) return;
  cudaFree(h->status);
  cudaFree(h->part_o);
  cudaFree(h->part_ml);
  cudaFree(h->counters);
  cudaFree(h->share_o);
  cudaFree(h->share_ml);
  cudaFree(h->own_o);
  cudaFree(h->own_ml);
  cudaFree(h->own_counters);
  delete h;
}

extern "C" tss_status tss_paged_sync_status(tss_paged* h, void* stream) {
  if (!h) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  const tss_status on = still_on(h->dev);
  if (on != TSS_OK) return on;
  int v = 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaMemcpyAsync(&v, h->status, sizeof(int), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaMemsetAsync(h->status, 0, sizeof(int), s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return refuse_cuda(e, "status read");
  if (v != TSS_OK) return refuse(v, "device status of the paged cache's calls");
  return TSS_OK;
}

extern "C" tss_status tss_paged_inject_timeout(tss_paged* h, int n_calls) {
  if (!h || n_calls < 0) return refuse(TSS_ERR_INVALID_ARG, "NULL argument or n_calls < 0");
  h->inject = n_calls;
  return TSS_OK;
}

extern "C" tss_status tss_paged_append(tss_paged* h, const tss_paged_cache* cache, int layer, const tss_paged_batch* batch, const void* k,
                                       const void* v, int64_t k_stride, int64_t v_stride, int dtype, void* stream) {
  return quant_call(h, cache, layer, batch, k, v, nullptr, nullptr, k_stride, v_stride, dtype, true, stream);
}

extern "C" tss_status tss_paged_read(tss_paged* h, const tss_paged_cache* cache, int layer, const tss_paged_batch* batch, void* k, void* v,
                                     int64_t k_stride, int64_t v_stride, int dtype, void* stream) {
  return quant_call(h, cache, layer, batch, nullptr, nullptr, k, v, k_stride, v_stride, dtype, false, stream);
}

namespace tss {
namespace {

// Checks a call of the attention and lays it out; *rows 0: nothing to do.
tss_status take_attention(const tss_paged* h, const tss_paged_cache* cache, int layer, const tss_paged_batch* batch, const tss_paged_attn* a,
                          PgAttnArgs* out, PgBatch* batch_out, long long* rows_out) {
  PgAttnArgs& p = *out;
  PgBatch& b = *batch_out;
  long long& rows = *rows_out;
  const tss_status st = take_batch(h, cache, layer, batch, &b, &rows);
  if (st != TSS_OK) return st;
  if (!a) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  if (a->dtype != TSS_DTYPE_BF16 && a->dtype != TSS_DTYPE_F16) return refuse(TSS_ERR_INVALID_ARG, "dtype must be bf16 or fp16");
  for (int i = 0; i < b.n_req; ++i)
    if (b.r[i].n > kPgMaxRows) return refuse(TSS_ERR_INVALID_ARG, "a request's block has more than 128 rows");
  if (!(a->scale > 0.f) || !(a->scale < INFINITY)) return refuse(TSS_ERR_INVALID_ARG, "scale must be positive and finite");
  if (a->window < 0 || a->n_sinks < 0) return refuse(TSS_ERR_INVALID_ARG, "window and n_sinks must be >= 0");
  if (rows == 0) return TSS_OK;
  if (!a->q || !a->out) return refuse(TSS_ERR_INVALID_ARG, "q or out is NULL");
  const int64_t width = static_cast<int64_t>(h->hq) * h->d;
  if (!aligned16(a->q) || !aligned16(a->out) || !good_stride(a->q_stride, width, a->dtype) || !good_stride(a->out_stride, width, a->dtype))
    return refuse(TSS_ERR_INVALID_ARG, "q and out must be 16-byte aligned, their row strides hold the heads and be multiples of 16 bytes");
  if ((a->lse && (reinterpret_cast<uintptr_t>(a->lse) & 3u)) || (a->mask && (reinterpret_cast<uintptr_t>(a->mask) & 7u)) ||
      (a->positions && (reinterpret_cast<uintptr_t>(a->positions) & 3u)))
    return refuse(TSS_ERR_INVALID_ARG, "lse, mask or positions is not aligned to its elements");
  p.hq = h->hq;
  p.hk = h->hk;
  p.d = h->d;
  p.n_pages = cache->n_pages;
  p.max_pages = cache->max_pages;
  p.pool = static_cast<const uint8_t*>(cache->layer[layer]);
  p.table = cache->table;
  p.q = a->q;
  p.out = a->out;
  p.lse = a->lse;
  p.qs = a->q_stride;
  p.os = a->out_stride;
  p.scale_log2 = a->scale * 1.4426950408889634f;
  p.window = a->window;
  p.sinks = a->window ? a->n_sinks : 0;
  p.is_half = a->dtype == TSS_DTYPE_F16;
  p.mask = reinterpret_cast<const unsigned long long*>(a->mask);
  p.positions = a->window ? a->positions : nullptr;
  p.status = h->status;
  p.share_o = h->share_o;
  p.share_ml = h->share_ml;
  return TSS_OK;
}

tss_status attention_launched(cudaError_t e, bool too_large) {
  if (too_large) return refuse(TSS_ERR_INVALID_ARG, "too many (page, head, row tile) units in one call");
  return e == cudaSuccess ? TSS_OK : refuse_cuda(e, "launch");
}

}  // namespace
}  // namespace tss

extern "C" tss_status tss_paged_attention(tss_paged* h, const tss_paged_cache* cache, int layer, const tss_paged_batch* batch,
                                          const tss_paged_attn* a, void* stream) {
  PgAttnArgs p{};
  PgBatch b;
  long long rows = 0;
  const tss_status st = take_attention(h, cache, layer, batch, a, &p, &b, &rows);
  if (st != TSS_OK || rows == 0) return st;
  bool too_large = false;
  const cudaError_t e = launch_paged_attention(h, p, b, static_cast<cudaStream_t>(stream), &too_large);
  return attention_launched(e, too_large);
}

extern "C" tss_status tss_paged_attention_shared(tss_paged* h, const tss_paged_cache* cache, int layer, const tss_paged_batch* batch,
                                                 const tss_paged_groups* groups, const tss_paged_attn* a, void* stream) {
  PgAttnArgs p{};
  PgBatch b;
  long long rows = 0;
  const tss_status st = take_attention(h, cache, layer, batch, a, &p, &b, &rows);
  if (st != TSS_OK) return st;
  if (!groups) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  if (groups->n_groups < 1 || groups->n_groups > b.n_req || !groups->n_req || !groups->shared)
    return refuse(TSS_ERR_INVALID_ARG, "n_groups in [1, the batch's n_req], n_req and shared are wanted");
  PgGroups g;
  g.n = groups->n_groups;
  int at = 0;
  for (int i = 0; i < g.n; ++i) {
    if (groups->n_req[i] < 1 || groups->n_req[i] > b.n_req - at) return refuse(TSS_ERR_INVALID_ARG, "the groups' requests must be the batch's");
    if (groups->shared[i] < 0) return refuse(TSS_ERR_INVALID_ARG, "shared must be >= 0");
    for (int j = at; j < at + groups->n_req[i]; ++j)
      if (b.r[j].n && b.r[j].first < groups->shared[i]) return refuse(TSS_ERR_INVALID_ARG, "shared exceeds a request's first token");
    g.reqs[i] = groups->n_req[i];
    g.shared[i] = groups->shared[i] / kPgTokens * kPgTokens;
    at += groups->n_req[i];
  }
  if (at != b.n_req) return refuse(TSS_ERR_INVALID_ARG, "the groups' requests must be the batch's");
  if (rows > h->share_rows) return refuse(TSS_ERR_INVALID_ARG, "more rows than the workspace was made for (shared_rows)");
  if (rows == 0) return TSS_OK;
  bool too_large = false;
  const cudaError_t e = launch_paged_attention_shared(h, p, b, g, static_cast<cudaStream_t>(stream), &too_large);
  return attention_launched(e, too_large);
}
