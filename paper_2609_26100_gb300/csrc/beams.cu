// Beam search's selection: of every group (a text's beams) the n_keep best continuations over beams and vocabulary.
//
//   value(b, t) = score_b + x_bt - ln sum_u exp x_bu,  largest first, ties to the lowest b vocab + t
//
// One pass over the logits.  A CTA holds a chunk of a row in registers.  The k-th largest of its threads' maxima is at most the
// chunk's k-th largest, and only k threads have elements above it, so a scan of the registers against it leaves few candidates,
// which are ranked by (value, index).  With them goes the chunk's sum of exponentials.  The last CTA of a group to arrive joins
// the rows' sums and picks from the chunks' sorted lists in the same way: first the k-th largest head, then what is above it.
//
// Between rows the order goes by the last bits of the rows' sums.  Terms are 2^((x - m) log2e), m the chunk's largest logit and
// log2e in two parts, sums are 64-bit from a thread's own on, and a chunk's n_keep largest terms are put in again in 64 bits (the
// fast exponential is off by 2^-22, which a few likely tokens would leave in the sum): values are right to about 1e-8, compared in
// 64 bits and rounded once.  The order of all sums is the elements', whatever their alignment: equal rows have equal values.
#include "ops.cuh"

struct tss_beam {
  int max_rows, vocab, max_keep, dev, sms;
  long long lists;    // chunks in all that fit
  int* status;        // device
  int* counters;      // device [max_rows]: chunks of each group that are done, zero between launches
  uint2* part;        // device [lists][max_keep]: a chunk's largest, (value's bits, token)
  double2* sums;      // device [lists]: (largest logit m, sum of e^(x - m))
};

namespace tss {
namespace {

constexpr int kBmThreads = 256, kBmWarps = kBmThreads / 32;
constexpr int kBmKeep = 128, kBmBeams = 64;
constexpr int kBmPool = 4096;     // candidates that the join holds at once
constexpr float kBmMost = 1e38f;  // logits from here on count as infinite, those from minus that on down as masked

struct BmParams {
  int beams, keep, vocab, end_token;
  int chunks, len;        // of a row; elements of a chunk (the last one may have fewer)
  long long stride;
  const void* logits;
  const float* score;
  const int* done;
  float* score_out;
  int *parent, *token;
  int* counters;
  uint2* part;
  double2* sums;
  int* status;
};

// Floats (doubles) as whole numbers of the same order; -0 counts as 0.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float float_of(uint32_t o) { return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ unsigned long long order_of(double x) {
  const unsigned long long b = static_cast<unsigned long long>(__double_as_longlong(x + 0.));
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ double double_of(unsigned long long o) {
  return __longlong_as_double(static_cast<long long>(o >> 63 ? o & 0x7fffffffffffffffull : ~o));
}
// (value, index): larger values first, then lower indices
__device__ __forceinline__ bool ahead(unsigned long long a, uint32_t ai, unsigned long long b, uint32_t bi) { return a > b || (a == b && ai < bi); }

__device__ __forceinline__ float bm_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// e^(x - m): the difference is exact for 16-bit logits, log2e in two parts
constexpr float kLog2eHi = 1.44269502162933349609f, kLog2eLo = 1.92596299112661746887e-8f;
__device__ __forceinline__ float bm_term(float x, float m) {
  const float d = x - m;
  return bm_ex2(fmaf(d, kLog2eHi, d * kLog2eLo));
}

// The first k of n entries (value, index) in shared memory, which has room for the next power of two from n on, in the order of
// `before`, to `put(rank, value, index)`; all threads.
template <typename Before, typename Put>
__device__ __forceinline__ void pick(unsigned long long* val, uint32_t* idx, int n, int k, Before before, Put put) {
  const int tid = threadIdx.x;
  __syncthreads();
  if (n <= kBmThreads) {  // by counting who comes before
    if (tid < n) {
      const unsigned long long v = val[tid];
      const uint32_t x = idx[tid];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += before(val[j], idx[j], v, x);
      if (rank < k) put(rank, v, x);
    }
  } else {  // bitonic sort
    int size = 2 * kBmThreads;
    while (size < n) size *= 2;
    for (int j = n + tid; j < size; j += kBmThreads) {
      val[j] = 0;
      idx[j] = 0xffffffffu;
    }
    for (int run = 2; run <= size; run *= 2)
      for (int step = run / 2; step > 0; step /= 2) {
        __syncthreads();
        for (int j = tid; j < size / 2; j += kBmThreads) {
          const int a = 2 * j - (j & (step - 1)), b = a + step;
          const unsigned long long va = val[a], vb = val[b];
          const uint32_t xa = idx[a], xb = idx[b];
          if (before(vb, xb, va, xa) == ((a & run) == 0)) {
            val[a] = vb, idx[a] = xb;
            val[b] = va, idx[b] = xa;
          }
        }
      }
    __syncthreads();
    for (int j = tid; j < min(n, k); j += kBmThreads) put(j, val[j], idx[j]);
  }
  __syncthreads();
}

struct BmShared {
  unsigned long long top[kBmThreads];  // the threads' maxima
  uint32_t top_idx[kBmThreads];
  double sum[kBmWarps];
  double again[kBmKeep];
  double base[kBmBeams];               // score - ln sum of each row
  float most[kBmWarps];
  int n, last;
};

// The k-th of the threads' own largest entries: at least k entries are at or before it (the last one where fewer than k have any).
__device__ __forceinline__ void bound_of(BmShared& sh, unsigned long long v, uint32_t x, int k, unsigned long long* tv, uint32_t* tx) {
  const int tid = threadIdx.x;
  sh.top[tid] = v;
  sh.top_idx[tid] = x;
  __syncthreads();
  int rank = 0;
  for (int j = 0; j < kBmThreads; ++j) rank += ahead(sh.top[j], sh.top_idx[j], v, x) || (sh.top[j] == v && sh.top_idx[j] == x && j < tid);
  __syncthreads();
  if (rank == k - 1) {
    sh.top[0] = v;
    sh.top_idx[0] = x;
  }
  __syncthreads();
  *tv = sh.top[0];
  *tx = sh.top_idx[0];
}

// A chunk of a live row: its largest entries and its sum.
template <typename T, int EPT>
__device__ __forceinline__ void bm_chunk(const BmParams& p, BmShared& sh, unsigned long long* val, uint32_t* idx, long long row, int chunk) {
  constexpr int VEC = 16 / sizeof(T), NV = EPT / VEC;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int e0 = chunk * p.len, n = min(p.len, p.vocab - e0);
  const T* src = static_cast<const T*>(p.logits) + row * p.stride + e0;
  const bool whole = (reinterpret_cast<uintptr_t>(src) & 15u) == 0;
  float x[EPT];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = (tid + i * kBmThreads) * VEC;
    if (whole && at + VEC <= n) {
      load_vec<T, VEC>(src + at, x + i * VEC);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[i * VEC + j] = at + j < n ? to_f32(src[at + j]) : -INFINITY;
    }
  }
  float most = -INFINITY;
  int where = 0;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    if (x[i] <= -kBmMost) x[i] = -INFINITY;
    bad |= !(x[i] < kBmMost);
    if (x[i] > most) {
      most = x[i];
      where = i;
    }
  }
  const auto token = [&](int i) { return static_cast<uint32_t>(e0 + (tid + i / VEC * kBmThreads) * VEC + i % VEC); };
  float m = most;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) sh.most[warp] = m;
  if (tid == 0) sh.n = 0;
  bad = __syncthreads_or(bad);
#pragma unroll
  for (int i = 0; i < kBmWarps; ++i) m = fmaxf(m, sh.most[i]);
  const long long list = row * p.chunks + chunk;
  if (bad || m == -INFINITY) {  // nothing to offer
    if (tid == 0) __stcg(p.sums + list, make_double2(0., bad ? NAN : 0.));
    if (tid < p.keep) __stcg(p.part + list * p.keep + tid, make_uint2(order_of(-INFINITY), 0u));
    return;
  }
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < EPT; ++i) s[i & 3] += bm_term(x[i], m);
  double sum = static_cast<double>(s[0] + s[1]) + static_cast<double>(s[2] + s[3]);
  // candidates
  unsigned long long tv;
  uint32_t tx;
  bound_of(sh, order_of(most), most > -INFINITY ? token(where) : 0xffffffffu, p.keep, &tv, &tx);
  const float least = float_of(static_cast<uint32_t>(tv));
#pragma unroll
  for (int i = 0; i < EPT; ++i)
    if (x[i] >= least && x[i] > -INFINITY) {
      const unsigned long long v = order_of(x[i]);
      const uint32_t t = token(i);
      if (!ahead(tv, tx, v, t)) {
        const int at = atomicAdd(&sh.n, 1);
        val[at] = v;
        idx[at] = t;
      }
    }
  __syncthreads();
  const int found = sh.n;
  pick(val, idx, found, p.keep, ahead, [&](int rank, unsigned long long v, uint32_t t) {
    __stcg(p.part + list * p.keep + rank, make_uint2(static_cast<uint32_t>(v), t));
    // the term again, in 64 bits
    const float y = float_of(static_cast<uint32_t>(v));
    sh.again[rank] = exp(static_cast<double>(y) - static_cast<double>(m)) - static_cast<double>(bm_term(y, m));
  });
  if (tid < min(found, p.keep)) sum += sh.again[tid];  // (by rank, so that the sum's order does not depend on timing)
  for (int r = found + tid; r < p.keep; r += kBmThreads) __stcg(p.part + list * p.keep + r, make_uint2(order_of(-INFINITY), 0u));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) sh.sum[warp] = sum;
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int i = 1; i < kBmWarps; ++i) sum += sh.sum[i];
    __stcg(p.sums + list, make_double2(static_cast<double>(m), sum));
  }
}

// The group's chunks are done: its best.
__device__ __forceinline__ void bm_join(const BmParams& p, BmShared& sh, unsigned long long* val, uint32_t* idx, int group) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row0 = static_cast<long long>(group) * p.beams;
  const int lists = p.beams * p.chunks;
  const double none = -static_cast<double>(INFINITY);
  // rows: score - ln sum
  for (int b = warp; b < p.beams; b += kBmWarps) {
    const float s = p.score ? __ldcg(p.score + row0 + b) : 0.f;
    const bool fine = s > -INFINITY && s < INFINITY;
    if (lane == 0 && !(s < INFINITY)) report(p.status, kStatusCheck);
    double base = none;
    if (fine && !(p.done && __ldcg(p.done + row0 + b))) {
      const double2* sums = p.sums + (row0 + b) * p.chunks;
      double ref = none, sum = 0.;
      for (int c = lane; c < p.chunks; c += 32) {
        const double2 x = __ldcg(sums + c);
        if (x.y != x.y) sum = x.y;  // (a NaN stays one)
        if (!(x.y > 0.)) continue;
        const double r = fmax(ref, x.x);
        sum = (sum == 0. ? 0. : sum * exp(ref - r)) + x.y * exp(x.x - r);
        ref = r;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const double r2 = __shfl_xor_sync(0xffffffffu, ref, o), s2 = __shfl_xor_sync(0xffffffffu, sum, o), r = fmax(ref, r2);
        sum = (ref > none ? sum * exp(ref - r) : sum) + (r2 > none ? s2 * exp(r2 - r) : s2);
        ref = r;
      }
      if (sum != sum) {
        if (lane == 0) report(p.status, kStatusCheck);
      } else if (sum > 0.) {
        base = static_cast<double>(s) - (ref + log(sum));
      }
    }
    if (lane == 0) sh.base[b] = base;
  }
  __syncthreads();
  // An entry of the lists goes by its place among them, a finished beam by lists * keep + beam.
  const uint2* part = p.part + row0 * p.chunks * p.keep;
  const auto value = [&](int list, int rank) { return order_of(sh.base[list / p.chunks] + static_cast<double>(float_of(__ldcg(part + list * p.keep + rank).x))); };
  const uint32_t finished = static_cast<uint32_t>(lists) * p.keep, of_row = static_cast<uint32_t>(p.chunks) * p.keep;
  const auto row_of = [&](uint32_t x) { return x >= finished ? x - finished : x / of_row; };
  // Equal values: the lower row; in a row the larger logit (which 64 bits of the value may not show), then the lower token.
  const auto first_of = [&](unsigned long long a, uint32_t ax, unsigned long long b, uint32_t bx) {
    if (a != b) return a > b;
    const uint32_t ar = row_of(ax), br = row_of(bx);
    if (ar != br || ax >= finished) return ar < br;
    const uint32_t av = __ldcg(part + ax).x, bv = __ldcg(part + bx).x;
    return av > bv || (av == bv && ax < bx);  // (places of a row go by token where logits are equal)
  };
  const unsigned long long nothing = order_of(none);
  const auto offers = [&](int list) { return sh.base[list / p.chunks] > none; };
  // what comes before the k-th of the threads' best heads, and before every list's k-th
  unsigned long long bv = nothing, lv = nothing;
  for (int l = tid; l < lists; l += kBmThreads)
    if (offers(l)) {
      bv = max(bv, value(l, 0));
      lv = max(lv, value(l, p.keep - 1));
    }
  unsigned long long tv;
  uint32_t tx;
  bound_of(sh, bv, 0u, p.keep, &tv, &tx);
  sh.top[tid] = lv;
  __syncthreads();
  for (int o = kBmThreads / 2; o > 0; o >>= 1) {
    if (tid < o) sh.top[tid] = max(sh.top[tid], sh.top[tid + o]);
    __syncthreads();
  }
  tv = max(max(tv, sh.top[0]), nothing + 1);
  // finished beams go on as they are
  int n = 0;  // entries in the pool; the first ones are the best so far
  if (tid == 0) sh.n = 0;
  __syncthreads();
  if (tid < p.beams && p.done && __ldcg(p.done + row0 + tid)) {
    const float s = p.score ? __ldcg(p.score + row0 + tid) : 0.f;
    if (s > -INFINITY && s < INFINITY) {
      const int at = atomicAdd(&sh.n, 1);
      val[at] = order_of(static_cast<double>(s));
      idx[at] = finished + tid;
    }
  }
  // Lists in turns of one a thread; where the pool could overflow, what it has is cut to the best and the bound raised.
  for (int l0 = 0; l0 < lists; l0 += kBmThreads) {
    const int l = l0 + tid;
    bool more = l < lists && offers(l);
    for (int r0 = 0; r0 < p.keep && __syncthreads_or(more); r0 += 8) {
      n = sh.n;
      __syncthreads();
      if (n > kBmPool - 8 * kBmThreads) {
        unsigned long long kept_v = 0;
        uint32_t kept_x = 0;
        bool kept = false;
        int at = 0;
        pick(val, idx, n, p.keep, first_of, [&](int rank, unsigned long long v, uint32_t x) {
          kept_v = v, kept_x = x, kept = true, at = rank;
        });
        if (kept) {
          val[at] = kept_v;
          idx[at] = kept_x;
        }
        if (tid == 0) sh.n = min(n, p.keep);
        __syncthreads();
        if (n >= p.keep) tv = max(tv, val[p.keep - 1]);
      }
      for (int r = r0; more && r < min(r0 + 8, p.keep); ++r) {
        const unsigned long long v = value(l, r);
        more = v >= tv;
        if (more) {
          const int to = atomicAdd(&sh.n, 1);
          val[to] = v;
          idx[to] = static_cast<uint32_t>(l) * p.keep + r;
        }
      }
    }
  }
  __syncthreads();
  n = sh.n;
  const long long out = static_cast<long long>(group) * p.keep;
  pick(val, idx, n, p.keep, first_of, [&](int rank, unsigned long long v, uint32_t x) {
    p.score_out[out + rank] = static_cast<float>(double_of(v));
    p.parent[out + rank] = static_cast<int>(row0) + static_cast<int>(row_of(x));
    p.token[out + rank] = x >= finished ? p.end_token : static_cast<int>(__ldcg(part + x).y);
  });
  for (int r = n + tid; r < p.keep; r += kBmThreads) {
    p.score_out[out + r] = -INFINITY;
    p.parent[out + r] = p.token[out + r] = -1;
  }
}

template <typename T, int EPT>
__global__ void __launch_bounds__(kBmThreads) beam_kernel(const __grid_constant__ BmParams p) {
  extern __shared__ __align__(16) uint8_t bm_dyn[];
  __shared__ BmShared sh;
  unsigned long long* val = reinterpret_cast<unsigned long long*>(bm_dyn);
  uint32_t* idx = reinterpret_cast<uint32_t*>(val + kBmPool);
  const int tid = threadIdx.x;
  const long long row = blockIdx.x / p.chunks;
  const int chunk = static_cast<int>(blockIdx.x - row * p.chunks), group = static_cast<int>(row / p.beams);
  griddep_wait();
  griddep_launch();
  const float s = p.score ? __ldcg(p.score + row) : 0.f;
  if (s > -INFINITY && s < INFINITY && !(p.done && __ldcg(p.done + row))) bm_chunk<T, EPT>(p, sh, val, idx, row, chunk);
  __syncthreads();
  if (tid == 0) {
    sh.last = atom_add_acq_rel_gpu(&p.counters[group], 1) == p.beams * p.chunks - 1;
    if (sh.last) atomicExch(&p.counters[group], 0);
  }
  __syncthreads();
  if (sh.last) bm_join(p, sh, val, idx, group);
}

constexpr int kBmSmem = kBmPool * 12;

template <typename T>
cudaError_t bm_launch(const BmParams& p, int ept, unsigned grid, cudaStream_t s) {
  switch (ept) {
    case 8: return launch_k(beam_kernel<T, 8>, dim3(grid), dim3(kBmThreads), kBmSmem, s, true, p);
    case 16: return launch_k(beam_kernel<T, 16>, dim3(grid), dim3(kBmThreads), kBmSmem, s, true, p);
    default: return launch_k(beam_kernel<T, 32>, dim3(grid), dim3(kBmThreads), kBmSmem, s, true, p);
  }
}
template <typename T>
cudaError_t bm_prepare() {
  cudaError_t e = cudaFuncSetAttribute(beam_kernel<T, 8>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBmSmem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(beam_kernel<T, 16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBmSmem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(beam_kernel<T, 32>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBmSmem);
  return e;
}

long long chunks_of(int vocab, int ept) { return (vocab + kBmThreads * ept - 1) / (kBmThreads * ept); }

}  // namespace
}  // namespace tss

using namespace tss;

extern "C" tss_status tss_beam_create(int max_rows, int vocab, int max_keep, tss_beam** out) {
  if (!out) return refuse(TSS_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (max_rows < 1 || max_rows > (1 << 20)) return refuse(TSS_ERR_INVALID_ARG, "max_rows must be in [1, 2^20]");
  if (vocab < 1 || vocab > (1 << 24)) return refuse(TSS_ERR_INVALID_ARG, "vocab must be in [1, 2^24]");
  if (max_keep < 1 || max_keep > kBmKeep) return refuse(TSS_ERR_INVALID_ARG, "max_keep must be in [1, 128]");
  int dev = 0, sms = 0;
  const tss_status st = this_device(&dev, &sms);
  if (st != TSS_OK) return st;
  tss_beam* h = new (std::nothrow) tss_beam{};
  if (!h) return refuse(TSS_ERR_OUT_OF_MEMORY, "no host memory");
  h->max_rows = max_rows;
  h->vocab = vocab;
  h->max_keep = max_keep;
  h->dev = dev;
  h->sms = sms;
  h->lists = max_rows * chunks_of(vocab, 32);
  if (h->lists < 4LL * sms) h->lists = 4LL * sms;
  cudaError_t e = bm_prepare<float>();
  if (e == cudaSuccess) e = bm_prepare<__half>();
  if (e == cudaSuccess) e = bm_prepare<__nv_bfloat16>();
  if (e == cudaSuccess) e = cudaMalloc(&h->status, 256);
  if (e == cudaSuccess) e = zero_now(h->status, 256);
  if (e == cudaSuccess) e = cudaMalloc(&h->counters, sizeof(int) * static_cast<size_t>(max_rows));
  if (e == cudaSuccess) e = zero_now(h->counters, sizeof(int) * static_cast<size_t>(max_rows));
  if (e == cudaSuccess) e = cudaMalloc(&h->part, sizeof(uint2) * static_cast<size_t>(h->lists) * max_keep);
  if (e == cudaSuccess) e = cudaMalloc(&h->sums, sizeof(double2) * static_cast<size_t>(h->lists));
  if (e != cudaSuccess) {
    tss_beam_destroy(h);
    const tss_status r = refuse_cuda(e, "workspace");
    return e == cudaErrorMemoryAllocation ? TSS_ERR_OUT_OF_MEMORY : r;
  }
  *out = h;
  return TSS_OK;
}

extern "C" void tss_beam_destroy(tss_beam* h) {
  if (!h) return;
  cudaFree(h->status);
  cudaFree(h->counters);
  cudaFree(h->part);
  cudaFree(h->sums);
  delete h;
}

extern "C" tss_status tss_beam_sync_status(tss_beam* h, void* stream) {
  if (!h) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  const tss_status on = still_on(h->dev);
  if (on != TSS_OK) return on;
  int v = 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaMemcpyAsync(&v, h->status, sizeof(int), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaMemsetAsync(h->status, 0, sizeof(int), s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return refuse_cuda(e, "status read");
  if (v != TSS_OK) return refuse(static_cast<tss_status>(v), "device status of the beam calls");
  return TSS_OK;
}

extern "C" tss_status tss_beam_select(tss_beam* h, const tss_beam_args* a, void* stream) {
  if (!h || !a) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  const tss_status on = still_on(h->dev);
  if (on != TSS_OK) return on;
  if (a->n_groups < 0 || a->n_beams < 1 || a->n_beams > kBmBeams) return refuse(TSS_ERR_INVALID_ARG, "n_groups >= 0 and n_beams in [1, 64] are wanted");
  if (a->n_keep < 1 || a->n_keep > h->max_keep) return refuse(TSS_ERR_INVALID_ARG, "n_keep must be in [1, max_keep]");
  const long long rows = static_cast<long long>(a->n_groups) * a->n_beams;
  if (rows > h->max_rows) return refuse(TSS_ERR_INVALID_ARG, "more rows than the workspace was made for");
  if (!known_dtype(a->dtype)) return refuse(TSS_ERR_INVALID_ARG, "unknown dtype");
  if (a->done && (a->end_token < 0 || a->end_token >= h->vocab)) return refuse(TSS_ERR_INVALID_ARG, "end_token must be in [0, vocab)");
  if (rows == 0) return TSS_OK;
  if (!a->logits || !a->score_out || !a->parent || !a->token) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  const uintptr_t el = dtype_bytes(a->dtype) - 1;
  const void* words[] = {a->score, a->done, a->score_out, a->parent, a->token};
  for (const void* w : words)
    if (reinterpret_cast<uintptr_t>(w) & 3u) return refuse(TSS_ERR_INVALID_ARG, "score, done and the outputs must be aligned to their elements");
  if (reinterpret_cast<uintptr_t>(a->logits) & el) return refuse(TSS_ERR_INVALID_ARG, "logits is not aligned to its elements");
  if (a->stride < h->vocab || a->stride >= (int64_t(1) << 40)) return refuse(TSS_ERR_INVALID_ARG, "the row stride must hold the vocabulary");
  BmParams p{};
  p.beams = a->n_beams;
  p.keep = a->n_keep;
  p.vocab = h->vocab;
  p.end_token = a->end_token;
  p.stride = a->stride;
  p.logits = a->logits;
  p.score = a->score;
  p.done = a->done;
  p.score_out = a->score_out;
  p.parent = a->parent;
  p.token = a->token;
  p.counters = h->counters;
  p.part = h->part;
  p.sums = h->sums;
  p.status = h->status;
  // Chunks of 2048, 4096 or 8192 elements: the smallest that give no more CTAs than two an SM.
  int ept = 8;
  while (ept < 32 && rows * chunks_of(h->vocab, ept) > 2LL * h->sms) ept *= 2;
  p.chunks = static_cast<int>(chunks_of(h->vocab, ept));
  p.len = (h->vocab + p.chunks - 1) / p.chunks;
  p.len = (p.len + 7) / 8 * 8;
  const long long grid = rows * p.chunks;
  if (grid > 0x7fffffffLL) return refuse(TSS_ERR_INVALID_ARG, "too many rows for one launch");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const unsigned g = static_cast<unsigned>(grid);
  const cudaError_t e = a->dtype == TSS_DTYPE_BF16  ? bm_launch<__nv_bfloat16>(p, ept, g, s)
                        : a->dtype == TSS_DTYPE_F16 ? bm_launch<__half>(p, ept, g, s)
                                                    : bm_launch<float>(p, ept, g, s);
  return e == cudaSuccess ? TSS_OK : refuse_cuda(e, "launch");
}
