// Beam search's selection: of every group (a text's beams) the n_keep best continuations over beams and vocabulary.
//
//   value(b, t) = score_b + x_bt - ln sum_u exp x_bu,  largest first, ties to the lowest b vocab + t
//
// One pass over the logits.  A CTA holds a chunk of a row in registers.  At least n_keep of its elements reach the least of its
// warps' ceil(n_keep / 8)-th largest thread maxima, and few more do: those are ranked by (value, index).  With them goes the
// chunk's sum of exponentials.  The last CTA of a group to arrive joins the rows' sums and picks from the chunks' sorted lists in
// the same way: a bound from one entry of each list, then what reaches it.
//
// Between rows the order goes by the last bits of the rows' sums.  Terms are 2^((x - m) log2e + f), m the chunk's largest logit,
// log2e in two parts, f what its product with m leaves of a whole number, so that chunks' sums differ by powers of two.  The
// candidates' terms, most of the sum, are computed to 2^-28 (the fast exponential's 2^-22 is for the others), and sums of
// threads are whole numbers, whose order does not matter: values are right to about 1e-8, compared in 64 bits and rounded once, and
// equal rows have equal values, whatever their alignment (elements go to threads by their index).
#include "ops.cuh"

struct tss_beam {
  int max_rows, vocab, max_keep, dev, sms;
  long long lists;    // chunks in all that fit
  int* status;        // device
  int* counters;      // device [max_rows]: chunks of each group that are done, zero between launches
  uint2* part;        // device [lists][max_keep]: a chunk's largest, (value's bits, token)
  longlong2* sums;    // device [lists]: sum of its terms in units of 2^(R - kBmBits); its largest logit m, and 2^32 if it has none to use
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
  longlong2* sums;
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

// e^x = 2^(R + t): R whole (of two floats, as it may pass 2^24) and of the chunk's largest logit m, t = (x - m) log2e + f.
constexpr float kLog2eHi = 1.44269502162933349609f, kLog2eLo = 1.92596299112661746887e-8f;
struct BmBase {
  float hi, lo, f;
  __device__ __forceinline__ explicit BmBase(float m) {
    const float t = m * kLog2eHi, rest = fmaf(m, kLog2eHi, -t) + m * kLog2eLo;
    hi = rintf(t);
    lo = rintf(rest);
    f = (t - hi) + (rest - lo);
  }
};
// 2^t by the fast exponential (2^-22 of it).
__device__ __forceinline__ float bm_term(float x, float m, float f) {
  const float d = x - m;
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(fmaf(d, kLog2eHi, fmaf(d, kLog2eLo, f))));
  return y;
}
// 2^t to about 2^-28 of it, times 2^kBmBits and rounded to a whole number: 2^n e^u with u in two floats, e^u = 1 + u + u^2 q(u).
constexpr int kBmBits = 37;  // 2^24 terms of up to 2 stay below 2^63
__device__ __forceinline__ long long bm_fixed(float x, float m, float f) {
  constexpr float kLn2Hi = 0.693147182464599609375f, kLn2Lo = -1.90465429995776804525e-9f;
  const float d = x - m, t = d * kLog2eHi, rest = fmaf(d, kLog2eHi, -t) + fmaf(d, kLog2eLo, f);
  const float n = rintf(t + rest), v = t - n;  // (exact)
  const float v1 = v + rest, v2 = rest - (v1 - v);
  const float u = v1 * kLn2Hi, w = fmaf(v1, kLn2Hi, -u) + fmaf(v1, kLn2Lo, v2 * kLn2Hi);
  float q = 1.f / 5040.f;
  q = fmaf(q, u, 1.f / 720.f);
  q = fmaf(q, u, 1.f / 120.f);
  q = fmaf(q, u, 1.f / 24.f);
  q = fmaf(q, u, 1.f / 6.f);
  q = fmaf(q, u, 0.5f);
  const float e = fmaf(u * u, q, fmaf(u, w, w));  // all but 1 + u
  if (n < -static_cast<float>(kBmBits) - 2.f) return 0;
  const float scale = __uint_as_float(static_cast<uint32_t>(static_cast<int>(n) + kBmBits + 127) << 23);
  return __float2ll_rn(scale) + __float2ll_rn(u * scale) + __float2ll_rn(e * scale);
}
__device__ __forceinline__ long long bm_fixed(float y) { return __float2ll_rn(y * static_cast<float>(1ll << kBmBits)); }

// The first k of n entries (value, index) in shared memory, which has room for the next power of two from n on, in the order of
// `before`, to `put(rank, value, index)`; all threads.
template <typename Before, typename Put>
__device__ __forceinline__ void pick(unsigned long long* val, uint32_t* idx, int n, int k, Before before, Put put) {
  const int tid = threadIdx.x;
  __syncthreads();
  if (n <= kBmThreads) {  // by counting who comes before: up to 8 threads an entry
    int per = 8;
    while (per > 1 && n * per > kBmThreads) per /= 2;
    const int e = tid / per, part = tid & (per - 1);
    unsigned long long v = 0;
    uint32_t x = 0;
    int rank = 0;
    if (e < n) {
      v = val[e];
      x = idx[e];
      for (int j = part; j < n; j += per) rank += before(val[j], idx[j], v, x);
    }
    for (int o = per / 2; o > 0; o /= 2) rank += __shfl_xor_sync(0xffffffffu, rank, o);
    if (e < n && part == 0 && rank < k) put(rank, v, x);
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
  unsigned long long top[kBmThreads];
  uint32_t top_idx[kBmThreads];
  long long sum[kBmWarps];
  double base[kBmBeams];               // score - ln sum of each row
  float most[kBmWarps], least[kBmWarps];
  unsigned long long bound[kBmWarps], last_of[kBmWarps];
  long long row_sum[kBmBeams];
  float2 row_base[kBmBeams];
  int n, last;
};

// The m-th largest of a warp's values, m in [1, 32] (in all lanes).
template <typename V>
__device__ __forceinline__ V nth_of(V v, int m, int lane) {
  int rank = 0;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const V o = __shfl_sync(0xffffffffu, v, j);
    rank += o > v || (o == v && j < lane);
  }
  return __shfl_sync(0xffffffffu, v, __ffs(__ballot_sync(0xffffffffu, rank == m - 1)) - 1);
}

// The k-th of the threads' own largest entries: at least k entries are at or before it, and no others than those threads' are
// before it.
__device__ __forceinline__ void bound_of(BmShared& sh, unsigned long long v, uint32_t x, int k, unsigned long long* tv, uint32_t* tx) {
  const int tid = threadIdx.x;
  __syncthreads();
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
  if (tid == 0) sh.n = 0;
  float mv[NV], most = -INFINITY;  // the vectors' maxima
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    mv[i] = x[i * VEC];
#pragma unroll
    for (int j = 1; j < VEC; ++j) mv[i] = fmaxf(mv[i], x[i * VEC + j]);
    most = fmaxf(most, mv[i]);
  }
  const auto token = [&](int i) { return static_cast<uint32_t>(e0 + (tid + i / VEC * kBmThreads) * VEC + i % VEC); };
  // A bound that at least n_keep elements reach: of every warp the ceil(n_keep / 8)-th largest of its threads' maxima, the least
  // of these.
  float m = most, least;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  least = p.keep <= kBmWarps ? m : nth_of(most, (p.keep + kBmWarps - 1) / kBmWarps, lane);
  if (lane == 0) {
    sh.most[warp] = m;
    sh.least[warp] = least;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kBmWarps; ++i) {
    m = fmaxf(m, sh.most[i]);
    least = fminf(least, sh.least[i]);
  }
  const long long list = row * p.chunks + chunk;
  uint2* part = p.part + list * p.keep;
  const auto offer_nothing = [&](bool bad) {
    if (tid == 0) __stcg(p.sums + list, make_longlong2(0, (bad ? 1ll << 32 : 0ll) | __float_as_uint(-INFINITY)));
    if (tid < p.keep) __stcg(part + tid, make_uint2(order_of(-INFINITY), 0u));
  };
  const BmBase base(m);
  // Elements that reach the bound become candidates, whose terms are added up apart; a NaN shows in the sum of the others.
  float s[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    const float y = bm_term(x[i], m, base.f);
    if (!(x[i] >= least)) s[i & 1] += y;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (mv[i] >= least) {
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (x[i * VEC + j] >= least && x[i * VEC + j] > -kBmMost) {
          const int at = atomicAdd(&sh.n, 1);
          if (at < kBmPool) {
            val[at] = order_of(x[i * VEC + j]);
            idx[at] = token(i * VEC + j);
          }
        }
    }
  const float odd = s[0] + s[1];
  if (__syncthreads_or(odd != odd || !(m < kBmMost)) || m <= -kBmMost) {
    // (where all are masked the difference from the largest is a NaN too)
    bool bad = !(m < kBmMost);
#pragma unroll
    for (int i = 0; i < EPT; ++i) bad |= x[i] != x[i];
    offer_nothing(__syncthreads_or(bad));
    return;
  }
  int found = sh.n;
  long long sum = bm_fixed(s[0]) + bm_fixed(s[1]);
  if (found > kBmPool / 4) {
    // Too many (a run of masked elements, or of equal ones): the n_keep-th of the threads' best is the bound, which n_keep
    // threads' elements reach at most; the candidates' terms are taken as the others' are.
    __syncthreads();  // (all have read how many)
    int where = 0;
    float s2 = 0.f;
#pragma unroll
    for (int i = EPT - 1; i >= 0; --i) {
      if (x[i] == most) where = i;
      if (x[i] >= least) s2 += bm_term(x[i], m, base.f);
    }
    sum += bm_fixed(s2);
    if (tid == 0) sh.n = 0;
    unsigned long long tv;
    uint32_t tx;
    bound_of(sh, order_of(most), most > -kBmMost ? token(where) : 0xffffffffu, p.keep, &tv, &tx);
    const float from = float_of(static_cast<uint32_t>(tv));
#pragma unroll
    for (int i = 0; i < EPT; ++i)
      if (x[i] >= from && x[i] > -kBmMost && !ahead(tv, tx, order_of(x[i]), token(i))) {
        const int at = atomicAdd(&sh.n, 1);
        val[at] = order_of(x[i]);
        idx[at] = token(i);
      }
    __syncthreads();
    found = sh.n;
  } else {
    for (int j = tid; j < found; j += kBmThreads) sum += bm_fixed(float_of(static_cast<uint32_t>(val[j])), m, base.f);
  }
  pick(val, idx, found, p.keep, ahead, [&](int rank, unsigned long long v, uint32_t t) { __stcg(part + rank, make_uint2(static_cast<uint32_t>(v), t)); });
  for (int r = found + tid; r < p.keep; r += kBmThreads) __stcg(part + r, make_uint2(order_of(-INFINITY), 0u));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) sh.sum[warp] = sum;
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int i = 1; i < kBmWarps; ++i) sum += sh.sum[i];
    __stcg(p.sums + list, make_longlong2(sum, __float_as_uint(m)));
  }
}

// The group's chunks are done: its best.
__device__ __forceinline__ void bm_join(const BmParams& p, BmShared& sh, unsigned long long* val, uint32_t* idx, int group) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row0 = static_cast<long long>(group) * p.beams;
  const int lists = p.beams * p.chunks;
  const double none = -static_cast<double>(INFINITY);
  // rows' sums: a warp takes every eighth row, its lanes chunks; the rows' first chunks are on their way together
  constexpr int kRows = kBmBeams / kBmWarps;
  const auto alive = [&](int b) {
    const float s = p.score ? __ldcg(p.score + row0 + b) : 0.f;
    return s > -INFINITY && s < INFINITY && !(p.done && __ldcg(p.done + row0 + b));
  };
  longlong2 first[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int b = warp + i * kBmWarps;
    first[i] = make_longlong2(0, __float_as_uint(-INFINITY));
    if (b < p.beams && lane < p.chunks && alive(b)) first[i] = __ldcg(p.sums + (row0 + b) * p.chunks + lane);
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int b = warp + i * kBmWarps;
    if (b >= p.beams) break;
    const bool on = alive(b);
    float m = -INFINITY;
    bool bad = false;
    for (int c = lane; c < p.chunks; c += 32) {
      const longlong2 x = c < 32 ? first[i] : on ? __ldcg(p.sums + (row0 + b) * p.chunks + c) : make_longlong2(0, __float_as_uint(-INFINITY));
      m = fmaxf(m, __uint_as_float(static_cast<uint32_t>(x.y)));
      bad |= x.y >> 32 != 0;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    bad = __any_sync(0xffffffffu, bad);
    const BmBase top(m);
    long long sum = 0;
    for (int c = lane; c < p.chunks; c += 32) {
      const longlong2 x = c < 32 ? first[i] : on ? __ldcg(p.sums + (row0 + b) * p.chunks + c) : make_longlong2(0, __float_as_uint(-INFINITY));
      if (x.x == 0) continue;
      const BmBase mine(__uint_as_float(static_cast<uint32_t>(x.y)));
      const float down = (top.hi - mine.hi) + (top.lo - mine.lo);  // (whole; below 2^24 exact, beyond that nothing is left)
      if (down < 62.f) {
        const int k = max(static_cast<int>(down), 0);
        sum += k > 0 ? (x.x + (1ll << (k - 1))) >> k : x.x;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) {
      sh.row_sum[b] = bad ? 0 : sum;
      sh.row_base[b] = make_float2(m, top.f);
      if (bad) report(p.status, kStatusCheck);
    }
  }
  __syncthreads();
  bool goes_on = false;  // the thread's row is finished and goes on as it is
  float score = 0.f;
  if (tid < p.beams) {
    score = p.score ? __ldcg(p.score + row0 + tid) : 0.f;
    if (!(score < INFINITY)) report(p.status, kStatusCheck);
    const bool fine = score > -INFINITY && score < INFINITY, done = p.done && __ldcg(p.done + row0 + tid);
    goes_on = fine && done;
    const long long sum = sh.row_sum[tid];
    // (ln sum e^x = m + ln(2^-f sum of the terms): what R is does not come in)
    const float2 top = sh.row_base[tid];
    const double lse = static_cast<double>(top.x) + (log(static_cast<double>(sum)) - (static_cast<double>(top.y) + kBmBits) * 0.6931471805599453);
    sh.base[tid] = !fine || done || sum == 0 ? none : static_cast<double>(score) - lse;
  }
  if (tid == 0) sh.n = 0;
  __syncthreads();
  // An entry of the lists goes by its place among them, a finished beam by lists * keep + beam.
  const uint2* part = p.part + row0 * p.chunks * p.keep;
  const auto value_of = [&](int list, uint32_t x) { return order_of(sh.base[list / p.chunks] + static_cast<double>(float_of(x))); };
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
  // A bound that at least n_keep entries reach, as in a chunk: of the lists' `deep`-th entries (lists go round the warps); and the
  // largest of their last ones.
  const int deep = min(p.keep, (2 * p.keep + lists - 1) / lists);
  const int nth = ((p.keep + deep - 1) / deep + kBmWarps - 1) / kBmWarps;
  unsigned long long tv = nothing, lv = nothing;
  const int mine = warp + lane * kBmWarps;
  for (int l = mine; l < lists; l += kBmThreads)
    if (offers(l)) {
      const uint32_t a = __ldcg(part + l * p.keep + deep - 1).x, z = __ldcg(part + l * p.keep + p.keep - 1).x;
      tv = max(tv, value_of(l, a));
      lv = max(lv, value_of(l, z));
    }
  tv = nth_of(tv, nth, lane);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) lv = max(lv, __shfl_xor_sync(0xffffffffu, lv, o));
  if (lane == 0) {
    sh.bound[warp] = tv;
    sh.last_of[warp] = lv;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kBmWarps; ++i) {
    tv = min(tv, sh.bound[i]);
    lv = max(lv, sh.last_of[i]);
  }
  tv = max(max(tv, lv), nothing + 1);
  int n = 0;  // entries in the pool
  if (goes_on) {
    const int at = atomicAdd(&sh.n, 1);
    val[at] = order_of(static_cast<double>(score));
    idx[at] = finished + tid;
  }
  // The lists' entries that reach it, four of a list at a time; where the pool could overflow, what it has is cut to the best and
  // the bound raised.
  constexpr int kStep = 4;
  for (int l0 = 0; l0 < lists; l0 += kBmThreads) {
    const int l = l0 + mine;
    bool more = l < lists && offers(l);
    for (int r0 = 0; r0 < p.keep && __syncthreads_or(more); r0 += kStep) {
      n = sh.n;
      __syncthreads();
      if (n > kBmPool - kStep * kBmThreads) {
        unsigned long long kept_v = 0;
        uint32_t kept_x = 0;
        bool kept = false;
        int at = 0;
        pick(val, idx, n, p.keep, first_of, [&](int rank, unsigned long long v, uint32_t x) { kept_v = v, kept_x = x, kept = true, at = rank; });
        if (kept) {
          val[at] = kept_v;
          idx[at] = kept_x;
        }
        if (tid == 0) sh.n = min(n, p.keep);
        __syncthreads();
        if (n >= p.keep) tv = max(tv, val[p.keep - 1]);
      }
      if (more) {
        uint32_t e[kStep];
#pragma unroll
        for (int r = 0; r < kStep; ++r) e[r] = r0 + r < p.keep ? __ldcg(part + l * p.keep + r0 + r).x : order_of(-INFINITY);
#pragma unroll
        for (int r = 0; r < kStep; ++r) {
          const unsigned long long v = value_of(l, e[r]);
          more = more && v >= tv;
          if (more) {
            const int to = atomicAdd(&sh.n, 1);
            val[to] = v;
            idx[to] = static_cast<uint32_t>(l) * p.keep + r0 + r;
          }
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
__global__ void __launch_bounds__(kBmThreads, 3) beam_kernel(const __grid_constant__ BmParams p) {
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
  if (e == cudaSuccess) e = cudaMalloc(&h->sums, sizeof(longlong2) * static_cast<size_t>(h->lists));
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
