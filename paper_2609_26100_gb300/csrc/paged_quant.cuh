// Quantising rows into 4-bit pages, for the calls that append (paged.cu, append_rope.cu).
//
// A warp takes one (request, 32-token half page, KV head, K or V).  A lane holds 8 neighbouring dims, a
// token D / 8 lanes, so a warp's load brings two (four) whole tokens.  Of four loads at a time the 8 lanes of a group
// exchange ranges so that each ends up with one token's, finds its scale and hands it round (one lane's
// work instead of eight's: 50 us instead of 58 for 7171 rows of 40 heads).  A lane's K codes of a token are one
// 32-bit word.  A word of V codes is 8 tokens of a dim: a lane gathers those of even or of odd tokens, 16 bits
// of each word, and swaps half of them with the lane of the same dims at the other parity.  All words of a half
// page lie in one warp, so tokens that the call does not bring keep their nibbles and no two warps write one word.
#pragma once

#include "paged.h"

namespace tss {

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
__device__ __forceinline__ long long pq_warp() { return static_cast<long long>(blockIdx.x) * (kPqThreads / 32) + (threadIdx.x >> 5); }
// The unit of warp w; false past the last one.
__device__ __forceinline__ bool pq_unit(const PqParams& p, long long w, int lane, PqUnit* u) {
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

// The tokens of a run: src, token u.lo's first element of the head, stride elements between tokens (of memory that the warp may
// read; 16-byte vectors).
template <typename T, int D>
__device__ __forceinline__ void quantise_run(const PqParams& p, PqUnit& u, const T* src, long long stride, int lane) {
  using B = PgBlock<D>;
  using L = PqLane<D>;
  const L at(lane);
  src += at.d0;
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

// Checks a call on the cache and lays out its batch (k, v, their strides and outputs are the caller's to set); *rows: rows in
// all.  pq_once: no sequence appears twice.
tss_status pq_take(const tss_paged* h, const tss_paged_cache* cache, int layer, const tss_paged_batch* batch, PqParams* p, long long* rows);
bool pq_once(const PgBatch& b);

}  // namespace tss
