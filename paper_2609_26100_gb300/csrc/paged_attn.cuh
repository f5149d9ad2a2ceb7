// What the two kernels of the paged attention share: the plan of a launch, the joining of partial results,
// the output of a row.
#pragma once

#include "paged.h"

namespace tss {

struct PaReq {
  int seq, first, n, row;
  int units;             // of one item: those in sight, [0, sink) and [lo, ...)
  int sink, lo;
  int off, items0;       // units of all items before the request; those items
  int cta, splits;       // aligned runs: CTAs before the request, CTAs of one item
};
struct PaParams {
  PgAttnArgs a;
  int n_req, total;      // units in all
  int aligned;           // a CTA's run lies within one item
  int halves;            // 32-token halves of a unit: 2 (a page) or 1
  int lead;              // even runs: units that an item counts beside its own, for its start and end
  int weight;            // even runs: units and leads in all
  int withhold;          // fault injection: the first CTA's first warp copies nothing, or its MMA warp issues none
  float* part_o;         // [grid][2][rows][D]
  float2* part_ml;       // [grid][2][rows]
  int* counters;         // [grid], zero between launches
  PaReq r[kPgMaxReq];
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The tcgen05 kernel (paged_attn_tc.cu; head_dim 128, planned with R = 128 and whole pages) and the query rows of a KV
// head above which a request goes there.  A page costs it the same for any number of rows, the warp-level kernel in
// proportion to its 16-row tiles; us, warp-level / tcgen05, four requests of 4600 tokens and 32 heads: 24 rows 66 / 103,
// 48 rows 97 / 110, 56 rows 119 / 111, 128 rows 225 / 123; 8 heads: 32 rows 28 / 40, 48 rows 33 / 42, 64 rows 41 / 42.
constexpr int kPaTcRows = 48;
cudaError_t paged_attn_tc_prepare();
cudaError_t launch_paged_attention_tc(PaParams& p, int sms, cudaStream_t s);

// The power of two that brings a row's largest query value `big` into [2^14, 2^15), where fp16 holds the row exactly
// (kept within what it and its use in 2^24 / it can be; 1 for a row of zeros, or with an infinity).
__device__ __forceinline__ float query_scale(float big) {
  const int e = min(100, max(-100, 14 - (static_cast<int>(__float_as_uint(big) >> 23) - 127)));
  return big > 0.f && big < INFINITY ? __uint_as_float(static_cast<uint32_t>(e + 127) << 23) : 1.f;
}

// p s' that raises a row's reference, and fp16's smallest scale.
constexpr float kTop = 32768.f;
constexpr float kLeast = 5.9604645e-8f;
// 2^d of a whole d below 128 (0 where that is less than fp32's normal numbers).
__device__ __forceinline__ float pow2(float d) { return d < -126.f ? 0.f : __int_as_float((static_cast<int>(d) + 127) << 23); }

// Two codes as fp16 subnormals (c 2^-24; c 2^-20 from nibbles four bits up) as c - 7.5 times 2^-9, exactly.  The tensor cores
// cut off what passes the end of an fp32 sum, where a subnormal counts as if it were 2^-14: sums of codes as they are, all
// positive, lose 2^-17 of themselves an MMA or more, always downwards (over a run of 16000 keys 1e-4 of the values' spread);
// centred ones are as right as fp32.
__device__ __forceinline__ uint32_t centre(uint32_t codes, bool up) {
  const __half2 mul = __half2half2(__ushort_as_half(up ? 0x6800 : 0x7800)), add = __half2half2(__ushort_as_half(0xa380));  // 2^11, 2^15; -7.5 2^-9
  const __half2 y = __hfma2(*reinterpret_cast<const __half2*>(&codes), mul, add);
  return *reinterpret_cast<const uint32_t*>(&y);
}

// Even runs.  The items' units, each item's led by p.lead more, laid end to end and cut evenly: the first unit at
// or after place g of them, and the CTA whose run holds unit u (of request b).
__device__ __forceinline__ int unit_at(const PaParams& p, int g) {
  int b = 0;
  while (b + 1 < p.n_req && p.r[b + 1].off + p.lead * p.r[b + 1].items0 <= g) ++b;
  const PaReq& r = p.r[b];
  const int v = g - r.off - p.lead * r.items0, item = v / (r.units + p.lead);
  return r.off + item * r.units + max(0, v - item * (r.units + p.lead) - p.lead);
}
__device__ __forceinline__ int cta_of_unit(const PaParams& p, int b, int u) {
  const PaReq& r = p.r[b];
  const int g = u + p.lead * (r.items0 + (u - r.off) / r.units + 1);
  const long long T = p.weight, G = gridDim.x;
  int c = static_cast<int>(g * G / T);
  while ((c + 1) * T / G <= g) ++c;
  return c;
}

// The CTA's run of units [u0, u1); of an aligned run, its item's first CTA and the number of them.
__device__ __forceinline__ void cta_run(const PaParams& p, int* u0, int* u1, int* first_cta, int* splits) {
  const int cta = blockIdx.x;
  if (p.aligned) {
    int b = 0;
    while (b + 1 < p.n_req && p.r[b + 1].cta <= cta) ++b;
    const PaReq& r = p.r[b];
    const int c = cta - r.cta, item = c / r.splits, j = c - item * r.splits, at = r.off + item * r.units;
    *u0 = at + static_cast<int>(static_cast<long long>(r.units) * j / r.splits);
    *u1 = at + static_cast<int>(static_cast<long long>(r.units) * (j + 1) / r.splits);
    *first_cta = cta - j;
    *splits = r.splits;
  } else {
    *u0 = unit_at(p, static_cast<int>(static_cast<long long>(p.weight) * cta / gridDim.x));
    *u1 = cta + 1 == static_cast<int>(gridDim.x) ? p.total : unit_at(p, static_cast<int>(static_cast<long long>(p.weight) * (cta + 1) / gridDim.x));
    *first_cta = *splits = 0;
  }
}

// Units of a request that every row of a tile sees: [0, *all0), the sinks', and [*all1, *all2); pmax: the last position
// among the rows.  (No difference here leaves 32 bits, whatever the window and the position.)
__device__ __forceinline__ void units_in_sight(const PgAttnArgs& a, const PaReq& r, int unit, int pmax, int* all0, int* all1, int* all2) {
  *all0 = a.window ? min(r.sink, a.sinks / unit) : 0;
  *all1 = r.sink + (a.window && pmax >= a.window ? max(0, (pmax - a.window) / unit + 1 - r.lo) : 0);
  *all2 = r.sink + r.first / unit - r.lo;
}

// One warp: the partials that CTAs c0 + slice, c0 + slice + step, ... up to c1 left of a row, joined: the
// reference and sum (in all lanes) and, in lane l < D / 4, dims 4 l .. 4 l + 3 of the unnormalised output.
// An item's first CTA left its part in its second slot, the others in their first.
template <int D>
__device__ __forceinline__ void gather_partials(const PaParams& p, int R, int c0, int c1, int row, int slice, int step, float* ref, float* sum,
                                                float4* out) {
  const int lane = threadIdx.x & 31, n = c1 - c0 + 1, mine = n > slice ? (n - slice + step - 1) / step : 0;
  const auto slot = [&](int k) {
    const int c = c0 + slice + k * step;
    return static_cast<long long>(c * 2 + (c == c0)) * R + row;
  };
  float2 ml;
  const auto fetch_ml = [&](int k) { ml = k < mine ? __ldcg(p.part_ml + slot(k)) : make_float2(-INFINITY, 0.f); };
  float4 y[8];
  const auto fetch = [&](int k) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      y[i] = k + i < mine && lane < D / 4 ? __ldcg(reinterpret_cast<const float4*>(p.part_o + slot(k + i) * D) + lane)
                                          : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  // (the first 32 references and the first 8 parts in flight together)
  fetch_ml(lane);
  fetch(0);
  float M = ml.x, L = 0.f;
  for (int k = lane + 32; k < mine; k += 32) M = fmaxf(M, __ldcg(p.part_ml + slot(k)).x);
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, x));
  const float mb = M == -INFINITY ? 0.f : M;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = 0; k0 < mine; k0 += 32) {
    if (k0 > 0) fetch_ml(k0 + lane);
    const float fw = k0 + lane < mine ? ex2(ml.x - mb) : 0.f;
    L = fmaf(fw, ml.y, L);
    const int m = min(32, mine - k0);
    for (int k = 0; k < m; k += 8) {
      if (k0 + k > 0) fetch(k0 + k);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = __shfl_sync(0xffffffffu, fw, (k + i) & 31);
        if (k + i >= m) continue;
        s.x = fmaf(x, y[i].x, s.x);
        s.y = fmaf(x, y[i].y, s.y);
        s.z = fmaf(x, y[i].z, s.z);
        s.w = fmaf(x, y[i].w, s.w);
      }
    }
  }
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) L += __shfl_xor_sync(0xffffffffu, L, x);
  *ref = M;
  *sum = L;
  *out = s;
}

// Four dims (from 4 c4) of the output of query row qr (token qr / group, query head of KV head h), and its lse.
template <int D>
__device__ __forceinline__ void finish_row(const PgAttnArgs& a, const PaReq& r, int h, int qr, int c4, float M, float L, float4 x) {
  const int gq = a.hq / a.hk;
  const float inv = L > 0.f ? 1.f / L : L == 0.f ? 0.f : L;  // (a NaN stays one)
  const float y[4] = {x.x * inv, x.y * inv, x.z * inv, x.w * inv};
  const long long tok = r.row + qr / gq;
  const int head = h * gq + qr % gq;
  const long long at = tok * a.os + static_cast<long long>(head) * D + c4 * 4;
  if (a.is_half)
    store_vec<__half, 4>(static_cast<__half*>(a.out) + at, y);
  else
    store_vec<__nv_bfloat16, 4>(static_cast<__nv_bfloat16*>(a.out) + at, y);
  if (c4 == 0 && a.lse) a.lse[tok * a.hq + head] = (M + log2f(L)) * 0.6931471805599453f;
}

// ------------------------------------------------------------------------------------------
// Host: the plan of a launch
// ------------------------------------------------------------------------------------------
// The requests of the batch that `take` picks, in row tiles of R query rows and units of `halves` 32-token
// halves; false where the units pass 2^30.
template <typename Take>
inline bool pa_plan(PaParams& p, const PgBatch& batch, Take take, int R, int halves) {
  const PgAttnArgs& a = p.a;
  const int unit = 32 * halves, gq = a.hq / a.hk;
  long long at = 0;
  int items = 0;
  p.halves = halves;
  p.n_req = 0;
  for (int i = 0; i < batch.n_req; ++i) {
    const PgReq& q = batch.r[i];
    if (q.n == 0 || !take(q)) continue;
    PaReq& r = p.r[p.n_req++];
    r = PaReq{q.seq, q.first, q.n, q.row, 0, 0, 0, static_cast<int>(at), items, 0, 1};
    const int end = (q.first + q.n + unit - 1) / unit;
    if (a.window) {
      r.lo = (q.first - a.window + 1 > 0 ? q.first - a.window + 1 : 0) / unit;
      const int sinks = a.sinks < q.first + q.n ? a.sinks : q.first + q.n;
      r.sink = (sinks + unit - 1) / unit;
      if (r.sink > r.lo) r.sink = r.lo;
    }
    r.units = r.sink + end - r.lo;
    const int mine = a.hk * ((q.n * gq + R - 1) / R);
    items += mine;
    at += static_cast<long long>(r.units) * mine;
    if (at > 0x1fffffff) return false;
  }
  p.total = static_cast<int>(at);
  return true;
}

// Cuts the units into runs for at most `most` CTAs and returns their number: even runs, every item counting `lead`
// units beside its own (for its start and end), or, where a CTA's run is then at most `slack` units longer, runs
// that lie within one item each (a CTA ends one item instead of two or three).  Runs have at least `least` units.
inline int pa_cut(PaParams& p, int most, int least, int slack, int lead) {
  const int even = (p.total + most - 1) / most;
  const auto items = [&](int i) { return ((i + 1 < p.n_req ? p.r[i + 1].off : p.total) - p.r[i].off) / p.r[i].units; };
  const auto ctas = [&](int len) {
    long long n = 0;
    for (int i = 0; i < p.n_req; ++i) n += static_cast<long long>(items(i)) * ((p.r[i].units + len - 1) / len);
    return n;
  };
  int run = even > least ? even : least;
  while (run <= even + slack && ctas(run) > most) ++run;
  p.aligned = run <= even + slack;
  if (!p.aligned) {
    p.lead = lead;
    p.weight = p.total + lead * (p.r[p.n_req - 1].items0 + items(p.n_req - 1));
    return p.total < most ? p.total : most;
  }
  int grid = 0;
  for (int i = 0; i < p.n_req; ++i) {
    p.r[i].cta = grid;
    p.r[i].splits = (p.r[i].units + run - 1) / run;
    grid += items(i) * p.r[i].splits;
  }
  return grid;
}

}  // namespace tss
