// Beam search's selection: of every group (a text's beams) the n_keep best continuations over beams and vocabulary.
//
//   value(b, t) = score_b + x_bt - ln sum_u exp x_bu,  largest first, ties to the lowest b vocab + t
//
// One pass over the logits.  A CTA takes a chunk of a row in tiles, the next one on its way while one is worked on.  A thread's part of
// a tile is a group, which leaves its largest element and its sum of exponentials.  At least n_keep elements reach the n_keep-th largest
// of the threads' largest (of up to 8: the least of the warps'): groups that reach it, few, are looked at again, an element a lane, and
// what reaches it is ranked by (value, index).  The last CTA of a group of beams to arrive joins the rows' sums and picks from the
// chunks' sorted lists in the same way: a bound from one entry of each list, then what reaches it.
//
// Bound: of large calls HBM while the CTAs read (6.5 TB/s until those of SMs with three are through; the exponentials take 11 of the 16
// places a cycle and SM), then the chunks' ends; 512 rows of 131072, bf16, 32 kept, 51 us in one wave of chunks of 16 tiles: 19 to 25 us of reading, 10 of a chunk's end (the bound
// 2.3, the groups' sums 2.3, the second look 4.3, the order 1.1), the last joins 13; in two waves of half as long chunks 59.5.  Of small
// ones chains of barriers: 4 rows of 32000 12.4 us (a chunk 4, the join 8), 64 of 50021, fp32, 19.6.
//
// Between rows the order goes by the last bits of the rows' sums.  Terms are 2^((x - m) log2e + f), m the chunk's largest logit,
// log2e in two parts, f what its product with m leaves of a whole number, so that chunks' sums differ by powers of two.  The
// candidates' terms are computed to 2^-27, the others' by the fast exponential (2^-22 of a term, and as much by its argument), in
// fp32 sums of a thread's (24 additions at most); sums of threads are whole numbers, whose order does not matter.  So ln sum and a
// value are off by less than 2^-19 (4e-7 at the most that was seen, fp32 rows of one value but for a few; 3e-8 where logits are many different
// numbers); rounding the value to fp32 leaves as much from 32 on.  Values are compared in 64 bits and rounded once, and equal rows of a call have
// equal values, whatever their alignment (elements go to threads by their index).
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
constexpr int kBmPool = 2048, kBmPoolOf = 1024;  // candidates that are held at once, by the join and by a chunk
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
// A CTA's dynamic shared memory: candidates (value, index); of a chunk's groups the largest element and the sum, in whose place comes
// the list of those that are looked at again.
constexpr int kBmTiles = 16, kBmGroups = kBmTiles * kBmThreads;
struct BmSpace {
  unsigned long long* val;
  uint32_t* idx;
  float *most, *sum;
  uint16_t* group;
  static constexpr int kBytes = kBmPoolOf * 12 + kBmGroups * 8;
  __device__ __forceinline__ BmSpace(uint8_t* at, int pool) {
    val = reinterpret_cast<unsigned long long*>(at);
    idx = reinterpret_cast<uint32_t*>(val + pool);
    most = reinterpret_cast<float*>(idx + pool);
    sum = most + kBmGroups;
    group = reinterpret_cast<uint16_t*>(sum);
  }
};
static_assert(kBmPool * 12 <= BmSpace::kBytes && kBmGroups <= 65536 && kBmTiles <= 32, "room for the join's, groups' numbers and a thread's mask");

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
__device__ __forceinline__ float bm_ex2(float t) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(t));
  return y;
}
__device__ __forceinline__ float bm_term(float x, float m, float f) {
  const float d = x - m;
  return bm_ex2(fmaf(d, kLog2eHi, fmaf(d, kLog2eLo, f)));
}
// 2^t to 2^-27 of it, times 2^kBmBits and rounded to a whole number: 2^n e^u with u in two floats, e^u = 1 + u + u^2 q(u) (what q leaves
// out is u^8 / 8!, at |u| = ln 2 / 2 5e-9).
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
// A sum relative to another base, of a larger logit: a shift, rounded.
__device__ __forceinline__ long long bm_down(long long sum, const BmBase& from, const BmBase& to) {
  const float down = (to.hi - from.hi) + (to.lo - from.lo);  // (whole; below 2^24 exact, beyond that nothing is left)
  if (!(down < 62.f)) return 0;
  const int k = max(static_cast<int>(down), 0);
  return k > 0 ? (sum + (1ll << (k - 1))) >> k : sum;
}
__device__ __forceinline__ long long bm_fixed(float y) { return __float2ll_rn(y * static_cast<float>(1ll << kBmBits)); }

// n entries (value, index) in shared memory, which has room for the next power of two from n on, in the order of `before` to
// `put(rank, value, index)`; all threads (one of the first 256 ranks goes to a thread at most).
template <typename Before, typename Put>
__device__ __forceinline__ void pick(unsigned long long* val, uint32_t* idx, int n, Before before, Put put) {
  const int tid = threadIdx.x;
  __syncthreads();
  if (n <= kBmThreads) {  // by counting who comes before: up to 8 threads an entry; indices only where values are equal
    int per = 8;
    while (per > 1 && n * per > kBmThreads) per /= 2;
    const int e = tid / per, part = tid & (per - 1);
    unsigned long long v = 0;
    int rank = 0, same = 0;
    if (e < n) {
      v = val[e];
#pragma unroll 4
      for (int j = part; j < n; j += per) {
        const unsigned long long o = val[j];
        rank += o > v;
        same += o == v;
      }
    }
    for (int o = per / 2; o > 0; o /= 2) {
      rank += __shfl_xor_sync(0xffffffffu, rank, o);
      same += __shfl_xor_sync(0xffffffffu, same, o);
    }
    if (e < n && part == 0) {
      const uint32_t x = idx[e];
      if (same > 1)
        for (int j = 0; j < n; ++j) rank += val[j] == v && before(v, idx[j], v, x);
      put(rank, v, x);
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
    for (int j = tid; j < n; j += kBmThreads) put(j, val[j], idx[j]);
  }
  __syncthreads();
}

// The pool's entries cut to the k best, in order; their number.
template <typename Before>
__device__ __forceinline__ int cut(unsigned long long* val, uint32_t* idx, int n, int k, int* count, Before before) {
  unsigned long long kept_v = 0;
  uint32_t kept_x = 0;
  int at = -1;
  pick(val, idx, n, before, [&](int rank, unsigned long long v, uint32_t x) {
    if (rank < k) kept_v = v, kept_x = x, at = rank;
  });
  if (at >= 0) {
    val[at] = kept_v;
    idx[at] = kept_x;
  }
  if (threadIdx.x == 0) *count = min(n, k);
  __syncthreads();
  return min(n, k);
}

struct BmShared {
  long long sum[kBmWarps];
  double base[kBmBeams];               // score - ln sum of each row
  long long row_sum[kBmBeams];
  float2 row_base[kBmBeams];           // its largest logit m, and f
  float2 near[kBmBeams];               // base in 32 bits, and how far off that may be
  float sorted[kBmWarps][32], most[kBmWarps], kth;
  float score[kBmBeams];
  int alive[kBmBeams];                 // 1: the row's logits count; 2: it is finished
  int n, groups, tiny, last;
};

// The k-th largest of the threads' values, k in [1, 256]: every warp sorts its own, and each finds its place among the others'.
// (The caller has a barrier before the next call.)
__device__ __forceinline__ float kth_of(BmShared& sh, float v, int k) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int run = 2; run <= 32; run *= 2)
#pragma unroll
    for (int step = run / 2; step > 0; step /= 2) {
      const float o = __shfl_xor_sync(0xffffffffu, v, step);
      v = ((lane & step) == 0) == ((lane & run) == 0) ? fmaxf(v, o) : fminf(v, o);  // (descending; the last run is of all)
    }
  sh.sorted[warp][lane] = v;
  __syncthreads();
  int rank = lane;
#pragma unroll
  for (int i = 1; i < kBmWarps; ++i) {
    const int w = (warp + i) % kBmWarps;
    int at = 0;  // of the warp's values those that come before
#pragma unroll
    for (int step = 16; step > 0; step /= 2) {
      const float o = sh.sorted[w][at + step - 1];
      if (o > v || (o == v && w < warp)) at += step;
    }
    const float o = sh.sorted[w][min(at, 31)];
    rank += at + (at < 32 && (o > v || (o == v && w < warp)));
  }
  if (rank == k - 1) sh.kth = v;
  __syncthreads();
  return sh.kth;
}

template <typename T>
struct Pair { using type = __half2; };
template <>
struct Pair<__nv_bfloat16> { using type = __nv_bfloat162; };

// A tile is EPT elements a thread, in vectors of 16 bytes that go round the threads; a thread's part of one is a group.
template <typename T, int EPT>
struct BmTile {
  static constexpr int VEC = 16 / sizeof(T), NV = EPT / VEC, kElems = kBmThreads * EPT;
  // Place in the tile of element i of thread tid's group.
  static __device__ __forceinline__ int at(int tid, int i) { return (tid + i / VEC * kBmThreads) * VEC + i % VEC; }
  // The group's elements of src, which has n, on their way; `whole`: src is aligned to 16 bytes.
  uint4 raw[NV];
  __device__ __forceinline__ void fetch(const T* src, int n, bool whole) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int a = at(threadIdx.x, i * VEC);
      if (whole && a + VEC <= n) {
        raw[i] = *reinterpret_cast<const uint4*>(src + a);
      } else {
        T t[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) t[j] = a + j < n ? src[a + j] : from_f32<T>(-INFINITY);
        memcpy(&raw[i], t, 16);
      }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    T t[VEC];
    memcpy(t, &raw[i / VEC], 16);
    return to_f32(t[i % VEC]);
  }
  // The largest (16-bit ones two at a time).
  __device__ __forceinline__ float most() const {
    if constexpr (sizeof(T) == 4) {
      float m = get(0);
#pragma unroll
      for (int i = 1; i < EPT; ++i) m = fmaxf(m, get(i));
      return m;
    } else {
      using T2 = typename Pair<T>::type;
      T2 t[NV * 4];
      memcpy(t, raw, sizeof(raw));
#pragma unroll
      for (int i = 1; i < NV * 4; ++i) t[0] = __hmax2(t[0], t[i]);
      return fmaxf(to_f32(t[0].x), to_f32(t[0].y));
    }
  }
};

// A chunk of a live row: its largest entries and its sum.
template <typename T, int EPT>
__device__ __forceinline__ void bm_chunk(const BmParams& p, BmShared& sh, const BmSpace& sp, long long row, int chunk) {
  using Tile = BmTile<T, EPT>;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int e0 = chunk * p.len, n_el = min(p.len, p.vocab - e0);
  const T* src = static_cast<const T*>(p.logits) + row * p.stride + e0;
  const bool whole = (reinterpret_cast<uintptr_t>(src) & 15u) == 0;
  if (tid == 0) sh.n = sh.groups = 0;
  // ---- the groups' largest elements, and their sums relative to them; the next tile is on its way meanwhile ----
  float best = -INFINITY;
  bool odd = false;
  int tiles = 0;
  Tile next;
  next.fetch(src, n_el, whole);
  for (int t0 = 0; t0 < n_el; t0 += Tile::kElems, ++tiles) {
    const Tile now = next;
    if (t0 + Tile::kElems < n_el) next.fetch(src + t0 + Tile::kElems, n_el - t0 - Tile::kElems, whole);
    const float g = now.most(), m = g > -kBmMost ? g : 0.f;
    const BmBase base(m);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (fabsf(m) < 1e6f) {  // (R is one float, and what x log2e loses is less than 2^-22 beside it)
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        const float x = now.get(i);
        s[i & 3] += bm_ex2(fmaf(x, kLog2eLo, fmaf(x, kLog2eHi, -base.hi)));
      }
    } else {
#pragma unroll
      for (int i = 0; i < EPT; ++i) s[i & 3] += bm_term(now.get(i), m, base.f);
    }
    const float sum = (s[0] + s[1]) + (s[2] + s[3]);
    sp.most[tiles * kBmThreads + tid] = g;
    sp.sum[tiles * kBmThreads + tid] = sum;
    best = fmaxf(best, g);
    odd |= sum != sum || !(g < kBmMost);
  }
  // ---- the chunk's largest, and a bound that at least n_keep elements reach: the n_keep-th largest of the threads' own, or, of
  // up to 8, the least of the warps' ----
  float m = best;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float least = m;
  if (lane == 0) sh.most[warp] = m;
  odd = __syncthreads_or(odd);
#pragma unroll
  for (int i = 0; i < kBmWarps; ++i) {
    m = fmaxf(m, sh.most[i]);
    least = fminf(least, sh.most[i]);
  }
  if (p.keep > kBmWarps) least = kth_of(sh, best, p.keep);
  const long long list = row * p.chunks + chunk;
  uint2* part = p.part + list * p.keep;
  if (odd || m <= -kBmMost) {  // nothing to offer
    if (tid == 0) __stcg(p.sums + list, make_longlong2(0, (odd ? 1ll << 32 : 0ll) | __float_as_uint(-INFINITY)));
    if (tid < p.keep) __stcg(part + tid, make_uint2(order_of(-INFINITY), 0u));
    return;
  }
  // ---- groups that reach the bound are looked at again, the others' sums added up ----
  const BmBase base(m);
  long long sum = 0;
  float others = 0.f;
  uint32_t again = 0;
  for (int t = 0; t < tiles; ++t) {
    const int id = t * kBmThreads + tid;
    const float g = sp.most[id];
    if (!(g > -kBmMost)) continue;
    if (g >= least)
      again |= 1u << t;
    else if (fabsf(g) < 1e6f && fabsf(m) < 1e6f)
      others = fmaf(sp.sum[id], bm_ex2(rintf(g * kLog2eHi) - base.hi), others);  // (a power of two)
    else
      sum += bm_down(bm_fixed(sp.sum[id]), BmBase(g), base);
  }
  sum += bm_fixed(others);
  __syncthreads();
  for (; again; again &= again - 1) sp.group[atomicAdd(&sh.groups, 1)] = static_cast<uint16_t>((__ffs(again) - 1) * kBmThreads + tid);
  __syncthreads();
  const int groups = sh.groups;
  // An element a lane: its term, and itself into the pool if it reaches the bound; where the pool could overflow it is cut to the
  // n_keep best, and others have to come before the last of them.
  constexpr int kAt = kBmThreads / EPT, kRound = 2, kFlight = 8;  // groups of a pass; passes of a round, and whose loads are in flight
  unsigned long long cv = 0;
  uint32_t cx = 0;
  int n = 0;
  for (int g0 = 0; g0 < groups; g0 += kAt * kFlight) {
    float x[kFlight];
    uint32_t at[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u) {
      const int g = g0 + u * kAt + tid / EPT;
      x[u] = -INFINITY;
      at[u] = 0;
      if (g < groups) {
        const int id = sp.group[g];
        at[u] = id / kBmThreads * Tile::kElems + Tile::at(id % kBmThreads, tid % EPT);
        if (static_cast<int>(at[u]) < n_el) x[u] = to_f32(src[at[u]]);
      }
    }
#pragma unroll
    for (int r = 0; r < kFlight; r += kRound) {
      if (g0 + kAt * r >= groups) break;
#pragma unroll
      for (int u = r; u < r + kRound; ++u) {
        if (!(x[u] > -kBmMost)) continue;
        sum += bm_fixed(x[u], m, base.f);
        const unsigned long long v = order_of(x[u]);
        if (x[u] >= least && !ahead(cv, cx, v, e0 + at[u])) {
          const int to = atomicAdd(&sh.n, 1);
          sp.val[to] = v;
          sp.idx[to] = e0 + at[u];
        }
      }
      __syncthreads();
      n = sh.n;
      if (g0 + kAt * (r + kRound) >= groups) break;
      __syncthreads();
      if (n > kBmPoolOf / 4) {
        n = cut(sp.val, sp.idx, n, p.keep, &sh.n, ahead);
        if (n == p.keep) {
          cv = sp.val[n - 1];
          cx = sp.idx[n - 1];
        }
        __syncthreads();
      }
    }
  }
  pick(sp.val, sp.idx, n, ahead, [&](int rank, unsigned long long v, uint32_t t) {
    if (rank < p.keep) __stcg(part + rank, make_uint2(static_cast<uint32_t>(v), t));
  });
  for (int r = n + tid; r < p.keep; r += kBmThreads) __stcg(part + r, make_uint2(order_of(-INFINITY), 0u));
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
__device__ __forceinline__ void bm_join(const BmParams& p, BmShared& sh, const BmSpace& sp, int group) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row0 = static_cast<long long>(group) * p.beams;
  const int lists = p.beams * p.chunks;
  const double none = -static_cast<double>(INFINITY);
  const uint2* part = p.part + row0 * p.chunks * p.keep;
  const longlong2* sums = p.sums + row0 * p.chunks;
  // The thread's first list's first entries, those that the bound comes from and the first chunks' sums are on their way together
  // (lists go round the warps; what rows without logits that count have left there is not used).
  constexpr int kStep = 4, kHead = 2 * kStep;
  const int deep = min(p.keep, (2 * p.keep + lists - 1) / lists), mine = warp + lane * kBmWarps;
  const auto entry = [&](int l, int r) { return l < lists && r < p.keep ? __ldcg(part + l * p.keep + r) : make_uint2(order_of(-INFINITY), 0u); };
  uint2 head[kHead];
#pragma unroll
  for (int r = 0; r < kHead; ++r) head[r] = entry(mine, r);
  const uint32_t deep_x = entry(mine, deep - 1).x, last_x = entry(mine, p.keep - 1).x;
  // (a row's chunks lie in `wide` lanes, a power of two)
  int wide = 1;
  while (wide < 32 && wide < p.chunks) wide *= 2;
  const int c0 = lane & (wide - 1), b0 = tid / wide, b_step = kBmThreads / wide;
  const auto sum_of = [&](int b, int c) { return b < p.beams && c < p.chunks ? __ldcg(sums + b * p.chunks + c) : make_longlong2(0, __float_as_uint(-INFINITY)); };
  longlong2 first = sum_of(b0, c0);
  if (tid < p.beams) {
    const float s = p.score ? __ldcg(p.score + row0 + tid) : 0.f;
    const int done = p.done ? __ldcg(p.done + row0 + tid) : 0;
    sh.score[tid] = s;
    sh.alive[tid] = !(s > -INFINITY && s < INFINITY) ? 0 : done ? 2 : 1;
    if (!(s < INFINITY)) report(p.status, kStatusCheck);
  }
  if (tid == 0) sh.n = sh.tiny = 0;
  __syncthreads();
  // ---- rows' sums ----
  for (int b_first = 0; b_first < p.beams; b_first += b_step) {
    const int b = b_first + b0;
    if (b_first > 0) first = sum_of(b, c0);
    const bool on = b < p.beams && sh.alive[b] == 1;
    float m = -INFINITY;
    bool bad = false;
    long long sum = 0;
    if (on)
      for (int c = c0; c < p.chunks; c += wide) {
        const longlong2 x = c == c0 ? first : sum_of(b, c);
        m = fmaxf(m, __uint_as_float(static_cast<uint32_t>(x.y)));
        bad |= x.y >> 32 != 0;
      }
    for (int o = wide / 2; o > 0; o /= 2) {
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      bad |= __shfl_xor_sync(0xffffffffu, static_cast<int>(bad), o);
    }
    const BmBase top(m);
    if (m > -kBmMost)
      for (int c = c0; c < p.chunks; c += wide) {
        const longlong2 x = c == c0 ? first : sum_of(b, c);
        if (x.x != 0) sum += bm_down(x.x, BmBase(__uint_as_float(static_cast<uint32_t>(x.y))), top);
      }
    for (int o = wide / 2; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (c0 == 0 && b < p.beams) {
      if (bad) sum = 0;
      sh.row_sum[b] = sum;
      sh.row_base[b] = make_float2(m, top.f);
      const float s = sh.score[b];
      sh.near[b] = sum > 0 ? make_float2(s - (m + (log2f(static_cast<float>(sum)) - top.f - kBmBits) * 0.69314718f), (fabsf(s) + fabsf(m) + 64.f) * 0x1p-20f)
                           : make_float2(-INFINITY, 0.f);
      if (bad) report(p.status, kStatusCheck);
    }
  }
  __syncthreads();
  // An entry goes by its place: row * of_row + chunk * keep + rank, a finished beam's by the row's last.
  const uint32_t in_row = static_cast<uint32_t>(p.chunks) * p.keep, of_row = in_row + 1;
  if (tid < p.beams) {
    // (ln sum e^x = m + ln(2^-f sum of the terms): what R is does not come in)
    const float2 top = sh.row_base[tid];
    const long long sum = sh.row_sum[tid];
    double base = none;
    if (sum > 0)
      base = static_cast<double>(sh.score[tid]) -
             (static_cast<double>(top.x) + (log(static_cast<double>(sum)) - (static_cast<double>(top.y) + kBmBits) * 0.6931471805599453));
    sh.base[tid] = base;
    if (sh.alive[tid] == 2) {  // a finished beam goes on as it is
      const int at = atomicAdd(&sh.n, 1);
      sp.val[at] = order_of(static_cast<double>(sh.score[tid]));
      sp.idx[at] = tid * of_row + in_row;
    }
  }
  // A bound that at least n_keep entries reach: of the lists' `deep`-th ones the ceil(n_keep / deep)-th largest, or the largest of
  // their last ones; of values in 32 bits, less what these may be off (64-bit logarithms take their time meanwhile).
  const auto least_of = [&](int l, uint32_t x) {
    const float2 b = sh.near[l / p.chunks];
    const float y = float_of(x);  // (of a row without logits that count whatever lay there, infinite or NaN too)
    return b.x > -INFINITY && y > -INFINITY ? (b.x + y) - (b.y + fabsf(y) * 0x1p-20f) : -INFINITY;
  };
  float tf = mine < lists ? least_of(mine, deep_x) : -INFINITY, lf = mine < lists ? least_of(mine, last_x) : -INFINITY;
  for (int l = mine + kBmThreads; l < lists; l += kBmThreads) {
    tf = fmaxf(tf, least_of(l, entry(l, deep - 1).x));
    lf = fmaxf(lf, least_of(l, entry(l, p.keep - 1).x));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) lf = fmaxf(lf, __shfl_xor_sync(0xffffffffu, lf, o));
  if (lane == 0) sh.most[warp] = lf;
  tf = kth_of(sh, tf, (p.keep + deep - 1) / deep);
#pragma unroll
  for (int i = 0; i < kBmWarps; ++i) tf = fmaxf(tf, sh.most[i]);
  const unsigned long long nothing = order_of(none);
  unsigned long long tv = max(order_of(static_cast<double>(tf)), nothing + 1);
  // Equal values: the lower row, then the lower token, which is the order of places; but where logits are so small that 64 bits of
  // a value may not show their difference, the larger one of a row first.
  const auto by_place = [](unsigned long long a, uint32_t ax, unsigned long long b, uint32_t bx) { return a > b || (a == b && ax < bx); };
  const auto by_logit = [&](unsigned long long a, uint32_t ax, unsigned long long b, uint32_t bx) {
    if (a != b || ax / of_row != bx / of_row || ax % of_row == in_row || ax == bx) return by_place(a, ax, b, bx);
    const uint32_t av = __ldcg(part + ax - ax / of_row).x, bv = __ldcg(part + bx - bx / of_row).x;
    return av > bv || (av == bv && ax < bx);
  };
  const auto sorted = [&](int n, auto put) {
    if (sh.tiny)
      pick(sp.val, sp.idx, n, by_logit, put);
    else
      pick(sp.val, sp.idx, n, by_place, put);
  };
  // ---- the lists' entries that reach it, a few of a list at a time; where the pool could overflow it is cut to the best and the
  // bound raised ----
  int n = 0;
  const auto take = [&](int l, int row, double base, int r, uint2 e, bool* more) {
    const unsigned long long v = order_of(base + static_cast<double>(float_of(e.x)));
    *more = *more && v >= tv;
    if (*more) {
      const int to = atomicAdd(&sh.n, 1);
      sp.val[to] = v;
      sp.idx[to] = static_cast<uint32_t>(l) * p.keep + r + row;
      const float y = fabsf(float_of(e.x));
      if (y < 1e-6f * fabsf(static_cast<float>(double_of(v)))) sh.tiny = 1;
    }
  };
  // (the same for all threads; n becomes what the pool has)
  const auto keep_room = [&](bool mine_more) {
    const bool any = __syncthreads_or(mine_more);
    n = sh.n;
    __syncthreads();
    if (n > kBmPool / 2) {
      unsigned long long kept_v = 0;
      uint32_t kept_x = 0;
      int at = -1;
      sorted(n, [&](int rank, unsigned long long v, uint32_t x) {
        if (rank < p.keep) kept_v = v, kept_x = x, at = rank;
      });
      if (at >= 0) {
        sp.val[at] = kept_v;
        sp.idx[at] = kept_x;
      }
      n = min(n, p.keep);
      if (tid == 0) sh.n = n;
      __syncthreads();
      if (n == p.keep) tv = max(tv, sp.val[n - 1]);
      __syncthreads();
    }
    return any;
  };
  static_assert(kStep * kBmThreads <= kBmPool / 2 && kBmWarps * kBmKeep <= kBmPool / 2, "room for a turn");
  for (int l0 = 0; l0 < lists; l0 += kBmThreads) {
    const int l = l0 + mine, row = l / p.chunks;
    const double base = l < lists ? sh.base[row] : none;
    bool more = base > none;
#pragma unroll
    for (int r0 = 0; r0 < kHead; r0 += kStep) {
      if (!keep_room(more)) break;
      if (more) {
#pragma unroll
        for (int r = r0; r < r0 + kStep; ++r) take(l, row, base, r, l0 > 0 ? entry(l, r) : head[r], &more);
      }
    }
    // what is left of a list is a warp's
    for (uint32_t rest = __ballot_sync(0xffffffffu, more && p.keep > kHead); keep_room(rest != 0); rest &= rest - 1) {
      if (rest == 0) continue;
      const int from = __shfl_sync(0xffffffffu, l, __ffs(rest) - 1), from_row = from / p.chunks;
      const double from_base = sh.base[from_row];
      for (int r = kHead + lane; r < p.keep; r += 32) {
        bool here = true;
        take(from, from_row, from_base, r, entry(from, r), &here);
      }
    }
  }
  const long long out = static_cast<long long>(group) * p.keep;
  sorted(n, [&](int rank, unsigned long long v, uint32_t x) {
    if (rank >= p.keep) return;
    const uint32_t row = x / of_row;
    p.score_out[out + rank] = static_cast<float>(double_of(v));
    p.parent[out + rank] = static_cast<int>(row0 + row);
    p.token[out + rank] = x - row * of_row == in_row ? p.end_token : static_cast<int>(__ldcg(part + x - row).y);
  });
  for (int r = n + tid; r < p.keep; r += kBmThreads) {
    p.score_out[out + r] = -INFINITY;
    p.parent[out + r] = p.token[out + r] = -1;
  }
}

// Tiles of 2048 elements (small calls) or of 16 KiB.
constexpr int kBmSmall = 8, kBmCtas = 4;
template <typename T, int EPT>
__global__ void __launch_bounds__(kBmThreads, kBmCtas) beam_kernel(const __grid_constant__ BmParams p) {
  extern __shared__ __align__(16) uint8_t bm_dyn[];
  __shared__ BmShared sh;
  const int tid = threadIdx.x;
  const long long row = blockIdx.x / p.chunks;
  const int chunk = static_cast<int>(blockIdx.x - row * p.chunks), group = static_cast<int>(row / p.beams);
  griddep_wait();
  griddep_launch();
  const float s = p.score ? __ldcg(p.score + row) : 0.f;
  if (s > -INFINITY && s < INFINITY && !(p.done && __ldcg(p.done + row))) bm_chunk<T, EPT>(p, sh, BmSpace(bm_dyn, kBmPoolOf), row, chunk);
  __syncthreads();
  if (tid == 0) {
    sh.last = atom_add_acq_rel_gpu(&p.counters[group], 1) == p.beams * p.chunks - 1;
    if (sh.last) atomicExch(&p.counters[group], 0);
  }
  __syncthreads();
  if (sh.last) bm_join(p, sh, BmSpace(bm_dyn, kBmPool), group);
}


template <typename T>
cudaError_t bm_launch(const BmParams& p, bool small, unsigned grid, cudaStream_t s) {
  return launch_k(small ? beam_kernel<T, kBmSmall> : beam_kernel<T, 64 / sizeof(T)>, dim3(grid), dim3(kBmThreads), BmSpace::kBytes, s, true, p);
}

long long chunks_of(int vocab, int len) { return (vocab + len - 1) / len; }

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
  h->lists = max_rows * chunks_of(vocab, 16 * kBmThreads);  // (the most that a call of fp32 logits has)
  if (h->lists < 2LL * sms) h->lists = 2LL * sms;
  cudaError_t e = cudaMalloc(&h->status, 256);
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
  // Chunks of a tile of 2048 elements where that makes two CTAs an SM at most.  Else of 1 to 16 tiles of 16 KiB: a CTA takes about
  // 1.2 us a tile, 3 us more and as many again for 32 kept, and an SM holds kBmCtas.
  int len = kBmSmall * kBmThreads;
  const bool small = rows * chunks_of(h->vocab, len) <= 2LL * h->sms;
  if (!small) {
    const int tile = 64 / dtype_bytes(a->dtype) * kBmThreads;
    const double start = 3. + a->n_keep / 10.;
    double least = 1e30;
    for (int t = 1; t <= kBmTiles; ++t) {
      const long long ctas = rows * chunks_of(h->vocab, t * tile), waves = (ctas + kBmCtas * h->sms - 1) / (kBmCtas * h->sms);
      const double us = waves * (start + 1.2 * t);
      if (us < least) {
        least = us;
        len = t * tile;
      }
    }
  }
  p.chunks = static_cast<int>(chunks_of(h->vocab, len));
  p.len = ((h->vocab + p.chunks - 1) / p.chunks + 7) / 8 * 8;
  const long long grid = rows * p.chunks;
  if (grid > 0x7fffffffLL) return refuse(TSS_ERR_INVALID_ARG, "too many rows for one launch");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const unsigned g = static_cast<unsigned>(grid);
  const cudaError_t e = a->dtype == TSS_DTYPE_BF16  ? bm_launch<__nv_bfloat16>(p, small, g, s)
                        : a->dtype == TSS_DTYPE_F16 ? bm_launch<__half>(p, small, g, s)
                                                    : bm_launch<float>(p, small, g, s);
  return e == cudaSuccess ? TSS_OK : refuse_cuda(e, "launch");
}
