// The paged 4-bit KV cache: its workspace, appending (quantising) tokens and reading them back.
//
// Quantisation, per token and 64 dims:  z = fp16(min), s = fp16((max - z) / 15), c = rint((x - z) / s).
// A warp takes one (request, 32-token half page, KV head, K or V).  A lane holds D / 32 neighbouring
// dims, so a token's row is one coalesced read and a group's minimum and maximum a butterfly over 16 or
// 32 lanes.  K codes are stored by token; V codes share a 32-bit word between 8 tokens of a dim, which the
// lane that owns the dim builds in registers (a half page's words all lie in one warp: tokens that the
// call does not bring keep their nibbles, and no two warps write one word).
//
// Bound: HBM for prompts (a token's 2 bytes a value in, half a byte out), latency for a step's few rows.
#include "paged.h"

namespace tss {
namespace {

constexpr int kPqThreads = 128;

struct PqParams {
  int hk, n_pages, max_pages, total;  // total: half pages touched by the batch
  uint8_t* pool;
  const int* table;
  const void *k, *v;
  void *ko, *vo;
  long long ks, vs;
  int* status;
  PgBatch batch;
  int off[kPgMaxReq + 1];  // half pages before each request
};

// The request that work unit u belongs to (the last one whose units begin at or before it).
__device__ __forceinline__ int owner_of(const int* off, int n, int u, int lane) {
  int b = 0;
#pragma unroll
  for (int i = 0; i < kPgMaxReq; i += 32) b += __popc(__ballot_sync(0xffffffffu, i + lane < n && off[i + lane] <= u));
  return b - 1;
}

struct PqUnit {
  int side, head, tok0, lo, hi;  // 32-token run of the page from token tok0; its tokens [lo, hi) are the batch's
  long long row;                 // row of token `lo` in the caller's arrays
  uint8_t* block;                // nullptr: the table's entry is no page
};
__device__ __forceinline__ bool pq_unit(const PqParams& p, int block_bytes, int lane, PqUnit* u) {
  const long long w = static_cast<long long>(blockIdx.x) * (kPqThreads / 32) + (threadIdx.x >> 5);
  const int per = 2 * p.hk;
  if (w >= static_cast<long long>(p.total) * per) return false;
  const int run = static_cast<int>(w / per), rest = static_cast<int>(w - static_cast<long long>(run) * per);
  u->side = rest & 1;
  u->head = rest >> 1;
  const int b = owner_of(p.off, p.batch.n_req, run, lane);
  const PgReq r = p.batch.r[b];
  const int half = r.first / 32 + run - p.off[b];  // 32-token run of the sequence
  const int t0 = half * 32;
  u->tok0 = t0 % kPgTokens;
  u->lo = max(r.first - t0, 0);
  u->hi = min(r.first + r.n - t0, 32);
  u->row = static_cast<long long>(r.row) + (t0 + u->lo - r.first);
  const int page = p.table[static_cast<long long>(r.seq) * p.max_pages + t0 / kPgTokens];
  u->block = nullptr;
  if (page >= 0 && page < p.n_pages)
    u->block = p.pool + (static_cast<long long>(page) * p.hk + u->head) * block_bytes;
  else if (lane == 0)
    report(p.status, kStatusCheck);
  return true;
}

// Scale and minimum of the group that the lane's N values belong to, and their codes.
template <int D, int N>
__device__ __forceinline__ __half2 quantise(const float* x, uint32_t* code) {
  float lo = x[0], hi = x[0];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
    bad |= !(fabsf(x[i]) < INFINITY);
  }
#pragma unroll
  for (int o = kPgGroup / N / 2; o > 0; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  // a NaN or an infinity poisons its group (one ballot; the group's lanes are neighbours)
  const uint32_t any = __ballot_sync(0xffffffffu, bad);
  constexpr int kLanes = kPgGroup / N;
  const int lane = threadIdx.x & 31;
  const uint32_t mine = kLanes == 32 ? 0xffffffffu : ((1u << (kLanes & 31)) - 1u) << (lane & ~(kLanes - 1));
  const __half z = __float2half_rn(fminf(fmaxf(lo, -65504.f), 65504.f));
  const float zf = __half2float(z);
  __half s = __float2half_rn(fminf(fmaxf(__fdiv_rn(__fsub_rn(hi, zf), 15.f), 0.f), 65504.f));
  const float sf = __half2float(s);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    // (the quotient is NaN or infinite only where s = 0 or the group is poisoned)
    const float c = sf > 0.f ? rintf(__fdiv_rn(__fsub_rn(x[i], zf), sf)) : 0.f;
    code[i] = static_cast<uint32_t>(fminf(fmaxf(c, 0.f), 15.f));
  }
  if (any & mine) {
    s = __ushort_as_half(0x7fff);
#pragma unroll
    for (int i = 0; i < N; ++i) code[i] = 0;
  }
  return __halves2half2(s, any & mine ? __ushort_as_half(0) : z);
}

// Byte of a K row that holds dims d, d + 1 (d even).
template <int D>
__device__ __forceinline__ int k_byte(int d) {
  return (d % kPgGroup) / 16 * (D / 8) + (d / kPgGroup) * 8 + (d % 16) / 2;
}

template <typename T, int D>
__global__ void __launch_bounds__(kPqThreads) append_kernel(const __grid_constant__ PqParams p) {
  using B = PgBlock<D>;
  constexpr int N = D / 32;  // dims of a lane
  const int lane = threadIdx.x & 31, d0 = lane * N;
  PqUnit u;
  if (!pq_unit(p, B::kBytes, lane, &u) || !u.block) return;
  const T* src = u.side ? static_cast<const T*>(p.v) + u.row * p.vs : static_cast<const T*>(p.k) + u.row * p.ks;
  const long long stride = u.side ? p.vs : p.ks;
  src += u.head * D + d0;
  const bool head = (d0 % kPgGroup) == 0;  // the lane that writes its group's parameters
  __half2* params = reinterpret_cast<__half2*>(u.block + (u.side ? B::kVParams : B::kKParams)) + u.tok0 * B::kGroups + d0 / kPgGroup;
  // the lane's V words: [t][dim]; those of a run that the batch fills only in part keep the other nibbles
  uint32_t words[4][N];
  uint32_t* vw = reinterpret_cast<uint32_t*>(u.block + B::kV) + ((u.tok0 / 32) * (D / 4) + d0 / 4) * 16 + d0 % 4;
  if (u.side && (u.lo > 0 || u.hi < 32)) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < N; ++e) words[t][e] = vw[t * 4 + e];
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < N; ++e) words[t][e] = 0u;
  }
#pragma unroll 1
  for (int b = u.lo / 8; b * 8 < u.hi; ++b) {
    float x[8][N];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int tok = 8 * b + i;
      if (tok >= u.lo && tok < u.hi) {
        load_vec<T, N>(src + (tok - u.lo) * stride, x[i]);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[i][e] = 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int tok = 8 * b + i;
      if (tok < u.lo || tok >= u.hi) continue;  // (the same for the whole warp)
      uint32_t c[N];
      const __half2 sz = quantise<D, N>(x[i], c);
      if (head) params[tok * B::kGroups] = sz;
      if (u.side) {
        const int shift = 4 * (b + 4 * (i & 1));
#pragma unroll
        for (int e = 0; e < N; ++e) words[i / 2][e] = (words[i / 2][e] & ~(15u << shift)) | (c[e] << shift);
      } else {
        uint8_t* dst = u.block + B::kK + (u.tok0 + tok) * (D / 2) + k_byte<D>(d0);
        if constexpr (N == 4)
          *reinterpret_cast<uint16_t*>(dst) = static_cast<uint16_t>(c[0] | c[1] << 4 | c[2] << 8 | c[3] << 12);
        else
          *dst = static_cast<uint8_t>(c[0] | c[1] << 4);
      }
    }
  }
  if (u.side) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if constexpr (N == 4)
        *reinterpret_cast<uint4*>(vw + t * 4) = make_uint4(words[t][0], words[t][1], words[t][2], words[t][3]);
      else
        *reinterpret_cast<uint2*>(vw + t * 4) = make_uint2(words[t][0], words[t][1]);
    }
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kPqThreads) read_kernel(const __grid_constant__ PqParams p) {
  using B = PgBlock<D>;
  constexpr int N = D / 32;
  const int lane = threadIdx.x & 31, d0 = lane * N;
  PqUnit u;
  if (!pq_unit(p, B::kBytes, lane, &u)) return;
  T* dst = static_cast<T*>(u.side ? p.vo : p.ko);
  if (!dst) return;
  const long long stride = u.side ? p.vs : p.ks;
  dst += u.row * stride + u.head * D + d0;
  const __half2* params = reinterpret_cast<const __half2*>(u.block + (u.side ? B::kVParams : B::kKParams)) + u.tok0 * B::kGroups + d0 / kPgGroup;
  const uint32_t* vw = reinterpret_cast<const uint32_t*>(u.block + B::kV) + ((u.tok0 / 32) * (D / 4) + d0 / 4) * 16 + d0 % 4;
  uint32_t words[4][N] = {};
  if (u.side && u.block) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < N; ++e) words[t][e] = vw[t * 4 + e];
  }
#pragma unroll 1
  for (int b = u.lo / 8; b * 8 < u.hi; ++b) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int tok = 8 * b + i;
      if (tok < u.lo || tok >= u.hi) continue;
      float x[N];
      if (!u.block) {  // no such page: zeros
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = 0.f;
      } else {
        const float2 sz = __half22float2(params[tok * B::kGroups]);
        uint32_t c;
        if (u.side) {
          const int shift = 4 * (b + 4 * (i & 1));
          c = 0;
#pragma unroll
          for (int e = 0; e < N; ++e) c |= ((words[i / 2][e] >> shift) & 15u) << (4 * e);
        } else {
          const uint8_t* s = u.block + B::kK + (u.tok0 + tok) * (D / 2) + k_byte<D>(d0);
          c = N == 4 ? *reinterpret_cast<const uint16_t*>(s) : *s;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = fmaf(static_cast<float>(c >> (4 * e) & 15u), sz.x, sz.y);
      }
      store_vec<T, N>(dst + (tok - u.lo) * stride, x);
    }
  }
}

template <int D>
void pq_launch(const PqParams& p, bool append, int dtype, unsigned grid, cudaStream_t s) {
#define TSS_PQ(T)                                      \
  if (append)                                          \
    append_kernel<T, D><<<grid, kPqThreads, 0, s>>>(p); \
  else                                                 \
    read_kernel<T, D><<<grid, kPqThreads, 0, s>>>(p)
  if (dtype == TSS_DTYPE_BF16) {
    TSS_PQ(__nv_bfloat16);
  } else if (dtype == TSS_DTYPE_F16) {
    TSS_PQ(__half);
  } else {
    TSS_PQ(float);
  }
#undef TSS_PQ
}

// Checks what every call on the cache has in common and copies the batch.  *rows: rows in all.
tss_status take_batch(const tss_paged* h, const tss_paged_cache* c, int layer, const tss_paged_batch* b, PgBatch* out, long long* rows) {
  if (!h || !c || !b) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
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

tss_status quant_call(tss_paged* h, const tss_paged_cache* cache, int layer, const tss_paged_batch* batch, const void* k, const void* v,
                      void* ko, void* vo, int64_t ks, int64_t vs, int dtype, bool append, void* stream) {
  PqParams p{};
  long long rows = 0;
  const tss_status st = take_batch(h, cache, layer, batch, &p.batch, &rows);
  if (st != TSS_OK) return st;
  if (!known_dtype(dtype)) return refuse(TSS_ERR_INVALID_ARG, "unknown dtype");
  if (append)
    for (int i = 0; i < p.batch.n_req; ++i)
      for (int j = 0; j < i; ++j)
        if (p.batch.r[i].seq == p.batch.r[j].seq) return refuse(TSS_ERR_INVALID_ARG, "a sequence appears twice");
  if (rows == 0) return TSS_OK;
  const int64_t width = static_cast<int64_t>(h->hk) * h->d;
  const void* ps[2] = {append ? k : ko, append ? v : vo};
  const int64_t strides[2] = {ks, vs};
  if (append ? (!ps[0] || !ps[1]) : (!ps[0] && !ps[1])) return refuse(TSS_ERR_INVALID_ARG, "k or v is NULL");
  for (int i = 0; i < 2; ++i)
    if (ps[i] && (!aligned16(ps[i]) || !good_stride(strides[i], width, dtype)))
      return refuse(TSS_ERR_INVALID_ARG, "k and v must be 16-byte aligned, their row strides hold the heads and be multiples of 16 bytes");
  long long total = 0;
  for (int i = 0; i < p.batch.n_req; ++i) {
    const PgReq& r = p.batch.r[i];
    p.off[i] = static_cast<int>(total);
    if (r.n) total += (r.first + r.n - 1) / 32 - r.first / 32 + 1;
  }
  p.total = static_cast<int>(total);
  p.hk = h->hk;
  p.n_pages = cache->n_pages;
  p.max_pages = cache->max_pages;
  p.pool = static_cast<uint8_t*>(cache->layer[layer]);
  p.table = cache->table;
  p.k = k;
  p.v = v;
  p.ko = ko;
  p.vo = vo;
  p.ks = ks;
  p.vs = vs;
  p.status = h->status;
  const long long warps = total * 2 * h->hk, per = kPqThreads / 32;
  if ((warps + per - 1) / per > 0x7fffffffLL) return refuse(TSS_ERR_INVALID_ARG, "too many rows for one launch");
  const unsigned grid = static_cast<unsigned>((warps + per - 1) / per);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (h->d == 64)
    pq_launch<64>(p, append, dtype, grid, s);
  else
    pq_launch<128>(p, append, dtype, grid, s);
  const cudaError_t e = cudaGetLastError();
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
  if (!out) return refuse(TSS_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (head_dim != 64 && head_dim != 128) return refuse(TSS_ERR_INVALID_ARG, "head_dim must be 64 or 128");
  if (n_kv_heads < 1 || n_kv_heads > 1024) return refuse(TSS_ERR_INVALID_ARG, "n_kv_heads must be in [1, 1024]");
  if (n_q_heads < 1 || n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > 64)
    return refuse(TSS_ERR_INVALID_ARG, "n_q_heads must be a multiple of n_kv_heads, at most 64 times it");
  int sms = 0;
  const tss_status st = this_device(&sms);
  if (st != TSS_OK) return st;
  tss_paged* h = new (std::nothrow) tss_paged{};
  if (!h) return refuse(TSS_ERR_OUT_OF_MEMORY, "no host memory");
  h->hq = n_q_heads;
  h->hk = n_kv_heads;
  h->d = head_dim;
  h->sms = sms;
  const size_t rows = pa_partial_rows(sms);
  cudaError_t e = pa_prepare_all();
  if (e == cudaSuccess) e = cudaMalloc(&h->status, 256);
  if (e == cudaSuccess) e = cudaMemset(h->status, 0, 256);
  if (e == cudaSuccess) e = cudaMalloc(&h->part_o, rows * head_dim * sizeof(float));
  if (e == cudaSuccess) e = cudaMalloc(&h->part_ml, rows * sizeof(float2));
  if (e == cudaSuccess) e = cudaMalloc(&h->counters, pa_counters(sms) * sizeof(int));
  if (e == cudaSuccess) e = cudaMemset(h->counters, 0, pa_counters(sms) * sizeof(int));
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
  delete h;
}

extern "C" tss_status tss_paged_sync_status(tss_paged* h, void* stream) {
  if (!h) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  int v = 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaMemcpyAsync(&v, h->status, sizeof(int), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaMemsetAsync(h->status, 0, sizeof(int), s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return refuse_cuda(e, "status read");
  if (v != TSS_OK) return refuse(v, "device status of the paged cache's calls");
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

extern "C" tss_status tss_paged_attention(tss_paged* h, const tss_paged_cache* cache, int layer, const tss_paged_batch* batch,
                                          const tss_paged_attn* a, void* stream) {
  PgAttnArgs p{};
  PgBatch b;
  long long rows = 0;
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
  bool too_large = false;
  const cudaError_t e = launch_paged_attention(h, p, b, static_cast<cudaStream_t>(stream), &too_large);
  if (too_large) return refuse(TSS_ERR_INVALID_ARG, "more than 2^30 (page, head, row tile) units in one call");
  return e == cudaSuccess ? TSS_OK : refuse_cuda(e, "launch");
}
