// The paged 4-bit KV cache: its workspace, appending (quantising) tokens and reading them back.
//
// Quantisation, per token and 64 dims:  z = fp16(min), s = fp16((max - z) / 15), c = rint((x - z) / s).
// A warp takes one (request, 32-token half page, KV head, K or V).  A lane holds 8 neighbouring dims, a
// token D / 8 lanes, so a warp's load brings two (four) whole tokens.  Of four loads at a time the 8 lanes of a group
// exchange ranges so that each ends up with one token's, finds its scale and hands it round (one lane's
// work instead of eight's: 50 us instead of 58 for 7171 rows of 40 heads).  A lane's K codes of a token are one
// 32-bit word.  A word of V codes is 8 tokens of a dim: a lane gathers those of even or of odd tokens, 16 bits
// of each word, and swaps half of them with the lane of the same dims at the other parity.  All words of a half
// page lie in one warp, so tokens that the call does not bring keep their nibbles and no two warps write one word.
//
// Bound: appending prompts, instruction issue (69 % of the slots, 17 instructions a value): 7171 rows of 40 heads of
// 128, bf16, 50 us, 3.8 TB/s of rows read and codes written.  Reading them back, HBM: 36 us, 5.2 TB/s.  A step's 16 rows:
// 4.4 us, launch and latency.
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
  int side, head, page, tok0, lo, hi;  // 32-token run of the page from token tok0; its tokens [lo, hi) are the batch's
  long long row;                 // row of token `lo` in the caller's arrays
  uint8_t* block;                // nullptr: the table's entry is no page
};
__device__ __forceinline__ bool pq_unit(const PqParams& p, int lane, PqUnit* u) {
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
  u->page = p.table[static_cast<long long>(r.seq) * p.max_pages + t0 / kPgTokens];
  return true;
}
// (apart, so that other loads can follow the table's before its answer is here)
__device__ __forceinline__ void pq_resolve(const PqParams& p, int block_bytes, int lane, PqUnit* u) {
  u->block = nullptr;
  if (u->page >= 0 && u->page < p.n_pages)
    u->block = p.pool + (static_cast<long long>(u->page) * p.hk + u->head) * block_bytes;
  else if (lane == 0)
    report(p.status, kStatusCheck);
}

// a / b rounded as by IEEE division, for a normal b whose reciprocal r approximates to a few ulp: the quotient by
// the reciprocal, corrected by its exact remainder (Markstein, IBM J. Res. Dev. 34, 1990).  A quotient that
// lies so near the middle of two floats that the rounded correction could miss its side would need more
// digits than a (24) and b (11 here) give.
__device__ __forceinline__ float quotient(float a, float b, float r) {
  const float q = a * r;
  return fmaf(fmaf(-b, q, a), r, q);
}

// Largest and negated smallest of the lane's 8 values; both not finite where one of them is not.  16-bit values two at a
// time, the two results in one register.
struct Range32 {
  float hi, nlo;
  __device__ __forceinline__ explicit Range32(const Raw8<float>& raw) {
    float x[8], odd = 0.f;
    raw.to(x);
    hi = x[0];
    nlo = -x[0];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      hi = fmaxf(hi, x[i]);
      nlo = fmaxf(nlo, -x[i]);
      odd = fmaf(x[i], 0.f, odd);  // NaN where a value is NaN or infinite
    }
    if (odd != 0.f) hi = INFINITY;
  }
  __device__ __forceinline__ void join(const Range32& give, int lanes) {
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, give.hi, lanes));
    nlo = fmaxf(nlo, __shfl_xor_sync(0xffffffffu, give.nlo, lanes));
  }
  __device__ __forceinline__ float2 both() const { return make_float2(hi, nlo); }
};
template <typename T, typename T2>
struct Range16 {
  T2 m;
  __device__ __forceinline__ explicit Range16(const Raw8<T>& raw) {
    T2 x[4];
    memcpy(x, raw.v, 16);
    const T2 a = __hmax2_nan(__hmax2_nan(x[0], x[1]), __hmax2_nan(x[2], x[3]));
    const T2 b = __hmax2_nan(__hmax2_nan(__hneg2(x[0]), __hneg2(x[1])), __hmax2_nan(__hneg2(x[2]), __hneg2(x[3])));
    uint32_t ab, bb;
    memcpy(&ab, &a, 4);
    memcpy(&bb, &b, 4);
    const uint32_t low = __byte_perm(ab, bb, 0x5410), high = __byte_perm(ab, bb, 0x7632);
    T2 c, d;
    memcpy(&c, &low, 4);
    memcpy(&d, &high, 4);
    m = __hmax2_nan(c, d);
  }
  __device__ __forceinline__ void join(const Range16& give, int lanes) { m = __hmax2_nan(m, __shfl_xor_sync(0xffffffffu, give.m, lanes)); }
  __device__ __forceinline__ float2 both() const { return make_float2(to_f32(m.x), to_f32(m.y)); }
};
template <typename T>
struct RangeOf;
template <>
struct RangeOf<float> { using type = Range32; };
template <>
struct RangeOf<__half> { using type = Range16<__half, __half2>; };
template <>
struct RangeOf<__nv_bfloat16> { using type = Range16<__nv_bfloat16, __nv_bfloat162>; };

// The groups of four tokens, 8 lanes and 64 dims each: a lane gets the range of token lane & 3 (each exchange halves the
// tokens that a lane goes on with), and from it that token's scale and minimum.  *inside: no quotient passes the codes'
// ends by as much as half a step (they do only where z's own rounding is worth that).
template <typename T>
__device__ __forceinline__ __half2 scale_of(const Raw8<T>* raw, int lane, bool* inside) {
  using R = typename RangeOf<T>::type;
  const R c0(raw[0]), c1(raw[1]), c2(raw[2]), c3(raw[3]);
  const bool odd = lane & 1, upper = lane & 2;
  R a = odd ? c1 : c0, b = odd ? c3 : c2;
  a.join(odd ? c0 : c1, 1);
  b.join(odd ? c2 : c3, 1);
  R m = upper ? b : a;
  m.join(upper ? a : b, 2);
  m.join(m, 4);
  const float2 range = m.both();
  const float hi = range.x, lo = -range.y;
  const __half z = __float2half_rn(fminf(fmaxf(lo, -65504.f), 65504.f));
  const float zf = __half2float(z);
  const __half s = __float2half_rn(fminf(fmaxf(quotient(hi - zf, 15.f, 1.f / 15.f), 0.f), 65504.f));
  const float sf = __half2float(s);
  if (!(fabsf(lo) < INFINITY && fabsf(hi) < INFINITY)) {  // a NaN or an infinity poisons its group
    *inside = true;
    return __halves2half2(__ushort_as_half(0x7fff), __ushort_as_half(0));
  }
  *inside = !(sf > 0.f) || (lo - zf > -0.49f * sf && hi - zf < 15.49f * sf);
  return __halves2half2(s, z);
}

// The codes of the lane's 8 values, one to a nibble; zeros where the scale is none.
template <typename T>
__device__ __forceinline__ uint32_t codes_of(const Raw8<T>& raw, __half2 sz, bool inside) {
  float x[8];
  raw.to(x);
  const float2 f = __half22float2(sz);
  const float sf = f.x, zf = f.y;
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(sf));
  // Rounded to an integer by adding 1.5 2^23: the low bits of the sum (ties to even, as rint).
  uint32_t w = 0;
  if (inside) {
    const f2_t nz = f2_pack(-zf, -zf), ns = f2_pack(-sf, -sf), r2 = f2_pack(r, r), magic = f2_pack(12582912.f, 12582912.f);
    const f2_t less = f2_pack(-12582912.f, -12582912.f), up = f2_pack(256.f, 256.f);
    f2_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f2_t d = f2_add(f2_pack(x[2 * i], x[2 * i + 1]), nz), q = f2_mul(d, r2);
      c[i] = f2_add(f2_add(f2_fma(f2_fma(ns, q, d), r2, q), magic), less);
    }
    // four codes to 16 bits by multiply-adds (c0 + 256 c2, c1 + 256 c3; the second times 16), as the low bits of 2^23 + n
    const float2 a = f2_unpack(f2_fma(c[1], up, c[0])), b = f2_unpack(f2_fma(c[3], up, c[2]));
    w = __byte_perm(__float_as_uint(fmaf(a.y, 16.f, a.x) + 8388608.f), __float_as_uint(fmaf(b.y, 16.f, b.x) + 8388608.f), 0x5410);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = fminf(fmaxf(quotient(x[i] - zf, sf, r), 0.f), 15.f);
      w |= (__float_as_uint(c + 12582912.f) & 15u) << (4 * i);
    }
  }
  return sf > 0.f ? w : 0u;
}

// Nibbles of word t of a run (token 8 b + 2 t + i at nibble b + 4 i) that are tokens [lo, hi).
__device__ __forceinline__ uint32_t word_mask(int t, int lo, int hi) {
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int tok = 8 * (k & 3) + 2 * t + (k >> 2);
    if (tok >= lo && tok < hi) m |= 15u << (4 * k);
  }
  return m;
}

template <int D>
struct PqLane {
  static constexpr int kLanes = D / 8;         // of a token
  static constexpr int kTokens = 32 / kLanes;  // of a warp's step: 2 or 4
  static constexpr int kT = 8 / kTokens;       // words (indices t) that a lane's tokens are spread over
  int d0, sub, i, k_at;
  __device__ explicit PqLane(int lane) {
    d0 = 8 * (lane % kLanes);
    sub = lane / kLanes;
    i = sub & 1;
    k_at = d0 % kPgGroup / 16 * (D / 8) + d0 / kPgGroup * 8 + d0 % 16 / 2;  // byte of the lane's word in a K row
  }
  // step j's token of the lane's is kTokens j + sub; its word t and nibble b + 4 i
  __device__ int t(int tl) const { return kTokens == 2 ? tl : 2 * tl + (sub >> 1); }
};

template <typename T, int D>
__global__ void __launch_bounds__(kPqThreads) append_kernel(const __grid_constant__ PqParams p) {
  using B = PgBlock<D>;
  using L = PqLane<D>;
  const int lane = threadIdx.x & 31;
  griddep_wait();
  griddep_launch();
  PqUnit u;
  if (!pq_unit(p, lane, &u)) return;
  const L at(lane);
  const T* src = u.side ? static_cast<const T*>(p.v) + u.row * p.vs : static_cast<const T*>(p.k) + u.row * p.ks;
  const long long stride = u.side ? p.vs : p.ks;
  src += u.head * D + at.d0;
  uint32_t acc[L::kT][4] = {};  // [t]: a byte for each even (odd) dim, nibbles b = 0, 1; the same of b = 2, 3
  constexpr int kStep = 4;      // steps whose loads are in flight together, and whose scales are found together
  Raw8<T> next[kStep];
  const auto fetch = [&](int j0) {
#pragma unroll
    for (int j = 0; j < kStep; ++j) {
      const int tok = (j0 + j) * L::kTokens + at.sub;
      if (tok >= u.lo && tok < u.hi)
        next[j].load(src + (tok - u.lo) * stride);
      else
        next[j].clear();
    }
  };
  const int first = u.lo / (kStep * L::kTokens) * kStep;
  fetch(first);
  pq_resolve(p, B::kBytes, lane, &u);
  if (!u.block) return;
  __half2* params = reinterpret_cast<__half2*>(u.block + (u.side ? B::kVParams : B::kKParams)) + u.tok0 * B::kGroups + at.d0 / kPgGroup;
  uint8_t* krow = u.block + B::kK + u.tok0 * (D / 2) + at.k_at;
#pragma unroll 1
  for (int j0 = first; j0 * L::kTokens < u.hi; j0 += kStep) {
    Raw8<T> now[kStep];
#pragma unroll
    for (int j = 0; j < kStep; ++j) now[j] = next[j];
    if ((j0 + kStep) * L::kTokens < u.hi) fetch(j0 + kStep);  // (on their way while these are worked on)
    bool inside;
    const __half2 scales = scale_of(now, lane, &inside);
    inside = __all_sync(0xffffffffu, inside);
#pragma unroll
    for (int j = 0; j < kStep; ++j) {
      const int tok0 = (j0 + j) * L::kTokens, tok = tok0 + at.sub;
      if (tok0 + L::kTokens <= u.lo || tok0 >= u.hi) continue;  // (the same for the whole warp)
      const __half2 sz = __shfl_sync(0xffffffffu, scales, (lane & 24) | j);
      const uint32_t w = codes_of(now[j], sz, inside);
      if (tok < u.lo || tok >= u.hi) continue;
      if (at.d0 % kPgGroup == 0) params[tok * B::kGroups] = sz;
      if (u.side) {
        const int b = tok0 / 8, shift = 4 * (b & 1);  // (the same for the whole warp)
        const uint32_t even = (w & 0x0f0f0f0fu) << shift, odd = (w >> 4 & 0x0f0f0f0fu) << shift;
        // (j0 is a multiple of kStep, a multiple of kT: the word is known at compile time)
        uint32_t(&to)[4] = acc[j % L::kT];
        if (b < 2) {
          to[0] |= even;
          to[1] |= odd;
        } else {
          to[2] |= even;
          to[3] |= odd;
        }
      } else {
        *reinterpret_cast<uint32_t*>(krow + tok * (D / 2)) = w;
      }
    }
  }
  if (!u.side) return;
  // to pairs of dims, 16 bits a dim, nibble b
#pragma unroll
  for (int t = 0; t < L::kT; ++t) {
    uint32_t(&x)[4] = acc[t];
    const uint32_t e0 = __byte_perm(x[0], x[2], 0x5140), e1 = __byte_perm(x[0], x[2], 0x7362);
    const uint32_t o0 = __byte_perm(x[1], x[3], 0x5140), o1 = __byte_perm(x[1], x[3], 0x7362);
    x[0] = __byte_perm(e0, o0, 0x5410);
    x[1] = __byte_perm(e0, o0, 0x7632);
    x[2] = __byte_perm(e1, o1, 0x5410);
    x[3] = __byte_perm(e1, o1, 0x7632);
  }
  // A lane of even tokens finishes the first half of its words, one of odd tokens the second.
  constexpr int kHalf = L::kT / 2;
#pragma unroll
  for (int h = 0; h < kHalf; ++h) {
    uint32_t lo16[4], hi16[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t keep = at.i ? acc[kHalf + h][e] : acc[h][e], give = at.i ? acc[h][e] : acc[kHalf + h][e];
      const uint32_t got = __shfl_xor_sync(0xffffffffu, give, L::kLanes);
      lo16[e] = at.i ? got : keep;  // even tokens: the words' low halves
      hi16[e] = at.i ? keep : got;
    }
    const int t = at.t(at.i * kHalf + h);
    const uint32_t mask = word_mask(t, u.lo, u.hi);
    if (mask == 0) continue;
    uint4* dst = reinterpret_cast<uint4*>(u.block + B::kV) + (u.tok0 / 32 * (D / 4) + at.d0 / 4) * 4 + t;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      uint4 v = make_uint4(__byte_perm(lo16[2 * q], hi16[2 * q], 0x5410), __byte_perm(lo16[2 * q], hi16[2 * q], 0x7632),
                           __byte_perm(lo16[2 * q + 1], hi16[2 * q + 1], 0x5410), __byte_perm(lo16[2 * q + 1], hi16[2 * q + 1], 0x7632));
      if (mask != 0xffffffffu) {
        const uint4 old = dst[4 * q];
        v.x |= old.x & ~mask;
        v.y |= old.y & ~mask;
        v.z |= old.z & ~mask;
        v.w |= old.w & ~mask;
      }
      dst[4 * q] = v;
    }
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kPqThreads) read_kernel(const __grid_constant__ PqParams p) {
  using B = PgBlock<D>;
  using L = PqLane<D>;
  const int lane = threadIdx.x & 31;
  griddep_wait();
  griddep_launch();
  PqUnit u;
  if (!pq_unit(p, lane, &u)) return;
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
  if (!out) return refuse(TSS_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (head_dim != 64 && head_dim != 128) return refuse(TSS_ERR_INVALID_ARG, "head_dim must be 64 or 128");
  if (n_kv_heads < 1 || n_kv_heads > 1024) return refuse(TSS_ERR_INVALID_ARG, "n_kv_heads must be in [1, 1024]");
  if (n_q_heads < 1 || n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > 64)
    return refuse(TSS_ERR_INVALID_ARG, "n_q_heads must be a multiple of n_kv_heads, at most 64 times it");
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
  if (e == cudaSuccess) e = cudaMalloc(&h->status, 256);
  if (e == cudaSuccess) e = zero_now(h->status, 256);
  if (e == cudaSuccess) e = cudaMalloc(&h->part_o, rows * head_dim * sizeof(float));
  if (e == cudaSuccess) e = cudaMalloc(&h->part_ml, rows * sizeof(float2));
  if (e == cudaSuccess) e = cudaMalloc(&h->counters, pa_counters(sms) * sizeof(int));
  if (e == cudaSuccess) e = zero_now(h->counters, pa_counters(sms) * sizeof(int));
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
  if (too_large) return refuse(TSS_ERR_INVALID_ARG, "too many (page, head, row tile) units in one call");
  return e == cudaSuccess ? TSS_OK : refuse_cuda(e, "launch");
}
