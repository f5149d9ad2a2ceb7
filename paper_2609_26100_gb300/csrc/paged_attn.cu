// Attention of draft blocks over the paged 4-bit cache, on warp-level tensor cores.
//
//   score_tr = scale q_r . k_t,  k_t = s_t c_t + z_t per 64 dims   (row r, token t)
//   o_r = sum_t p_tr v_t / sum_t p_tr,  p_tr = 2^(log2e score_tr - ref_r),  v_t = s'_t c'_t + z'_t
//
// The codes go to the tensor cores as they are: a nibble in the low bits of an fp16 lane is the subnormal
// number c 2^-24 (c 2^-20 four bits further up), so a 32-bit word becomes four operand registers with four
// ANDs and a shift, exactly; the factor 16 of every second pair is taken out of the other operand.  Scales
// and minima join in fp32: s_t multiplies the sum over a group's dims, z_t the sum of the query's; on the
// value side s'_t goes into the weight, which enters as two fp16 parts (hi and the rest, 22 bits: one part
// alone costs the output 4e-4 of its size, as much again as rounding it to fp16), and z'_t is summed by
// itself.  Queries are scaled by a power of two to fill fp16's range, so they are exact too.
//
// Tokens take the MMA's 16-row side (S^T = K Q^T, O^T = V^T P^T): a block of 8 query rows (N) fills it,
// where the usual orientation would pad 1 .. 8 rows to 16.  P^T's operand layout is the transpose of S^T's
// accumulator: one movmatrix per 8 x 8.
//
// ref_r is raised only when some p s' passes 2^15 (fp16's end), to where the largest is 2^7, so most tiles
// need no reduction over tokens.  In terms of p s' rather than p, it keeps the weights in fp16's range
// whatever the values' scales.
//
// Work split: the pages of all (request, row tile, KV head) items laid end to end and cut evenly, one CTA
// per SM.  A CTA's pages go round its warps, each with its own ring of bulk copies (a page of a head is one
// contiguous block, 9 KiB at head_dim 128).  At an item's end the warps' parts are joined in shared memory;
// items that several CTAs share leave partials, which the last one to arrive joins in CTA order.
#include <type_traits>

#include "paged.h"

namespace tss {
namespace {

struct PaReq {
  int seq, first, n, row;
  int pages, sink, lo;   // pages in sight: [0, sink) and [lo, ...); their number
  int off;               // units (page, head, row tile) before the request
};
struct PaParams {
  PgAttnParams a;        // (batch unused)
  int n_req, total;      // units in all
  float* part_o;         // [grid][2][rows][D]
  float2* part_ml;       // [grid][2][rows]
  int* counters;         // [grid], zero between launches
  PaReq r[kPgMaxReq];
};

__device__ __forceinline__ uint32_t movmatrix_t(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

constexpr float kTop = 32768.f;         // p s' that raises the reference
constexpr float kLeast = 5.9604645e-8f; // fp16's smallest scale

template <int D, int NT>
struct PaShape {
  static constexpr int kRows = 8 * NT;
  static constexpr int kWarps = NT == 1 ? 12 : 8;
  static constexpr int kStages = NT == 1 ? 2 : 3;
  static constexpr int kRing = kWarps * kStages * PgBlock<D>::kBytes;
  static constexpr size_t kSmem = kRing + 128;
};

// Whether row i (position qp, mask words anc or null) of request r sees key j.
__device__ __forceinline__ bool sees(const PgAttnParams& a, const PaReq& r, int i, int qp, const unsigned long long* anc, int j) {
  if (j >= r.first + r.n) return false;
  int kp = j;
  if (j >= r.first) {
    const int x = j - r.first;
    if (anc ? !(__ldg(anc + (x >> 6)) >> (x & 63) & 1ull) : x > i) return false;
    if (a.positions) kp = max(__ldg(a.positions + r.row + x), r.first);
  }
  return !a.window || qp - kp < a.window || j < a.sinks;
}

template <int D, int NT>
__global__ void __launch_bounds__(PaShape<D, NT>::kWarps * 32, 1) paged_attn_kernel(const __grid_constant__ PaParams p) {
  using B = PgBlock<D>;
  using S = PaShape<D, NT>;
  constexpr int G = B::kGroups, W = S::kWarps, ST = S::kStages, R = S::kRows, DB = D / 32;
  extern __shared__ uint8_t pa_dyn[];
  __shared__ uint64_t bars[W][ST];
  __shared__ int s_off[kPgMaxReq], s_pages[kPgMaxReq], s_sink[kPgMaxReq], s_lo[kPgMaxReq], s_seq[kPgMaxReq];
  __shared__ float2 s_ml[W][R];
  __shared__ int s_has[W], abort_s, s_last;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  uint8_t* ring_all = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(pa_dyn) + 127) & ~uintptr_t(127));
  uint8_t* ring = ring_all + warp * (ST * B::kBytes);
  const PgAttnParams& a = p.a;
  const int gq = a.hq / a.hk;
  const int u0 = static_cast<int>(static_cast<long long>(p.total) * blockIdx.x / gridDim.x);
  const int u1 = static_cast<int>(static_cast<long long>(p.total) * (blockIdx.x + 1) / gridDim.x);
  if (tid < p.n_req) {
    s_off[tid] = p.r[tid].off;
    s_pages[tid] = p.r[tid].pages;
    s_sink[tid] = p.r[tid].sink;
    s_lo[tid] = p.r[tid].lo;
    s_seq[tid] = p.r[tid].seq;
  }
  if (lane == 0)
    for (int i = 0; i < ST; ++i) mbar_init(&bars[warp][i], 1);
  if (tid == 0) abort_s = 0;
  fence_mbar_init();
  __syncthreads();
  volatile int* abort = &abort_s;

  const int mine = u0 + warp < u1 ? (u1 - u0 - warp + W - 1) / W : 0;  // the warp's units: u0 + warp + k W
  const auto request_of = [&](int u) {
    int b = 0;
#pragma unroll
    for (int s = kPgMaxReq / 2; s > 0; s >>= 1)
      if (b + s < p.n_req && s_off[b + s] <= u) b += s;
    return b;
  };
  // Lane l: block of unit k0 + l in the pool; -1 where the table names no page, -2 past the end.
  const auto blocks_from = [&](int k0) -> long long {
    if (k0 + lane >= mine) return -2;
    const int u = u0 + warp + (k0 + lane) * W, b = request_of(u), v = u - s_off[b];
    const int item = v / s_pages[b], pg = v - item * s_pages[b];
    const int h = item % a.hk, at = pg < s_sink[b] ? pg : pg - s_sink[b] + s_lo[b];
    const int page = __ldg(a.table + static_cast<long long>(s_seq[b]) * a.max_pages + at);
    if (page < 0 || page >= a.n_pages) {
      report(a.status, kStatusCheck);
      return -1;
    }
    return static_cast<long long>(page) * a.hk + h;
  };
  long long ids = blocks_from(0), ids_next = blocks_from(32);
  int ids_at = 0, issued = 0;
  uint32_t no_page = 0;  // bit s: stage s's unit has no page
  const auto issue = [&]() {  // the warp's next unit into stage issued % ST
    if (issued >= mine) return;
    if (issued - ids_at == 32) {
      ids = ids_next;
      ids_at += 32;
      ids_next = blocks_from(ids_at + 32);
    }
    const long long blk = __shfl_sync(0xffffffffu, ids, issued - ids_at);
    const int s = issued % ST;
    if (blk < 0) {
      no_page |= 1u << s;
      if (lane == 0) mbar_arrive(&bars[warp][s]);
    } else {
      no_page &= ~(1u << s);
      if (lane == 0) {
        mbar_arrive_expect_tx(&bars[warp][s], B::kBytes);
        bulk_load(ring + s * B::kBytes, a.pool + blk * B::kBytes, B::kBytes, &bars[warp][s]);
      }
    }
    ++issued;
  };
#pragma unroll
  for (int i = 0; i < ST; ++i) issue();

  int done = 0;  // the warp's units processed
  bool ok = true;
  for (int u = u0; u < u1;) {
    // ---- a segment: this CTA's pages [pg0, pg1) of an item ----
    const int b = request_of(u);
    const PaReq& r = p.r[b];
    const int v = u - r.off, item = v / r.pages, pg0 = v - item * r.pages;
    const int seg_end = min(u1, u - pg0 + r.pages), pg1 = pg0 + seg_end - u;
    const int h = item % a.hk, row0 = item / a.hk * R, rows = min(R, r.n * gq - row0);
    // Q: thread (g, t) holds row g's dims 64 gi + 16 t .. + 15 as the operand of 4 k-steps a group: pairs
    // (0, 4), (1, 5) and (2, 6), (3, 7) of each 8 dims, odd ones / 16 (their codes stand four bits up)
    uint32_t qf[NT][G][2][4];
    float f[NT][2], zq[NT][G][2], ref[NT][2], l[NT][2], oz[NT][G][2], o[NT][DB][2][4];
    int pmax = 0;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int qr = row0 + nt * 8 + g;
      float x[G][16], big = 0.f;
#pragma unroll
      for (int gi = 0; gi < G; ++gi) {
        if (nt * 8 + g < rows) {
          const long long at = (r.row + qr / gq) * a.qs + static_cast<long long>(h * gq + qr % gq) * D + gi * kPgGroup + 16 * t;
          if (a.is_half)
            load_vec<__half, 16>(static_cast<const __half*>(a.q) + at, x[gi]);
          else
            load_vec<__nv_bfloat16, 16>(static_cast<const __nv_bfloat16*>(a.q) + at, x[gi]);
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) x[gi][i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) big = fmaxf(big, fabsf(x[gi][i]));
      }
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
      // 2^e big in [2^14, 2^15); e kept within what 2^e and 2^(24 - e) can be
      const int e = min(100, max(-100, 14 - (static_cast<int>(__float_as_uint(big) >> 23) - 127)));
      const float up = big > 0.f && big < INFINITY ? __uint_as_float(static_cast<uint32_t>(e + 127) << 23) : 1.f;
      const float mul = a.scale_log2 * 16777216.f / up;
      float sum[G];
#pragma unroll
      for (int gi = 0; gi < G; ++gi) {
        sum[gi] = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[gi] += x[gi][i];
        sum[gi] += __shfl_xor_sync(0xffffffffu, sum[gi], 1);
        sum[gi] += __shfl_xor_sync(0xffffffffu, sum[gi], 2);
        sum[gi] *= a.scale_log2;
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float m = i & 1 ? up * 0.0625f : up;
            qf[nt][gi][w][i] = pack_f16(x[gi][8 * w + i] * m, x[gi][8 * w + i + 4] * m);
          }
      }
      // the accumulators' rows of a thread are 2t and 2t + 1
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int from = (2 * t + i) * 4;
        f[nt][i] = __shfl_sync(0xffffffffu, mul, from);
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
          zq[nt][gi][i] = __shfl_sync(0xffffffffu, sum[gi], from);
          oz[nt][gi][i] = 0.f;
        }
        ref[nt][i] = -INFINITY;
        l[nt][i] = 0.f;
      }
#pragma unroll
      for (int x2 = 0; x2 < DB; ++x2)
#pragma unroll
        for (int i = 0; i < 8; ++i) o[nt][x2][i >> 2][i & 3] = 0.f;
    }
    if (a.window) {  // the last position among the tile's rows
      if (lane < rows) {
        const int i = (row0 + lane) / gq;
        pmax = a.positions ? max(__ldg(a.positions + r.row + i), r.first) : r.first + i;
      }
#pragma unroll
      for (int x2 = 16; x2 > 0; x2 >>= 1) pmax = max(pmax, __shfl_xor_sync(0xffffffffu, pmax, x2));
    }
    const int done0 = done;
    for (int uu = u0 + warp + done * W; uu < seg_end; uu += W) {
      if (done > 0 && ok) issue();  // into the stage of the unit before this one
      const int s = done % ST;
      ok = __all_sync(0xffffffffu, ok && mbar_wait(&bars[warp][s], (done / ST) & 1, abort, a.status));
      ++done;
      if (!ok || (no_page >> s & 1u)) continue;
      const int pg = uu - u + pg0, key0 = (pg < r.sink ? pg : pg - r.sink + r.lo) * kPgTokens;
      const uint8_t* blk = ring + s * B::kBytes;
#pragma unroll 1
      for (int kg = 0; kg < 2; ++kg) {
        const int kb = key0 + 32 * kg;
        // every row sees all 32 keys?
        const bool full = kb + 32 <= r.first && (!a.window || kb > pmax - a.window || kb + 32 <= a.sinks);
        if (kb >= r.first + r.n) break;
        float sc[NT][2][4];  // scores: [16-key tile][key g, rows 2t and 2t + 1; key g + 8, the same]
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
          float acc[NT][G][4];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int gi = 0; gi < G; ++gi)
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[nt][gi][i] = 0.f;
          uint32_t kw[2][G][2];
#pragma unroll
          for (int x2 = 0; x2 < 2; ++x2) {
            const uint8_t* kp = blk + B::kK + (kg * 32 + mt * 16 + x2 * 8 + g) * (D / 2) + t * (D / 8);
            if constexpr (G == 2) {
              const uint4 w = *reinterpret_cast<const uint4*>(kp);
              kw[x2][0][0] = w.x, kw[x2][0][1] = w.y, kw[x2][G - 1][0] = w.z, kw[x2][G - 1][1] = w.w;
            } else {
              const uint2 w = *reinterpret_cast<const uint2*>(kp);
              kw[x2][0][0] = w.x, kw[x2][0][1] = w.y;
            }
          }
#pragma unroll
          for (int gi = 0; gi < G; ++gi)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              const uint32_t x0 = kw[0][gi][w], x1 = kw[1][gi][w], y0 = x0 >> 8, y1 = x1 >> 8;
              const uint32_t a0[4] = {x0 & 0x000f000fu, x1 & 0x000f000fu, x0 & 0x00f000f0u, x1 & 0x00f000f0u};
              const uint32_t a1[4] = {y0 & 0x000f000fu, y1 & 0x000f000fu, y0 & 0x00f000f0u, y1 & 0x00f000f0u};
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma_f16_16816(acc[nt][gi], a0, &qf[nt][gi][w][0]);
                mma_f16_16816(acc[nt][gi], a1, &qf[nt][gi][w][2]);
              }
            }
          // scores from the codes' sums
#pragma unroll
          for (int x2 = 0; x2 < 2; ++x2) {
            const __half2* pr = reinterpret_cast<const __half2*>(blk + B::kKParams) + (kg * 32 + mt * 16 + x2 * 8 + g) * G;
            float2 sz[G];
#pragma unroll
            for (int gi = 0; gi < G; ++gi) sz[gi] = __half22float2(pr[gi]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                float c = 0.f, z = 0.f;
#pragma unroll
                for (int gi = 0; gi < G; ++gi) {
                  c = fmaf(sz[gi].x, acc[nt][gi][2 * x2 + i], c);
                  z = fmaf(sz[gi].y, zq[nt][gi][i], z);
                }
                sc[nt][mt][2 * x2 + i] = fmaf(c, f[nt][i], z);
              }
          }
        }
        float2 vz[2][2][G];
        float smax[2][2];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int x2 = 0; x2 < 2; ++x2) {
            const __half2* pr = reinterpret_cast<const __half2*>(blk + B::kVParams) + (kg * 32 + mt * 16 + x2 * 8 + g) * G;
            smax[mt][x2] = kLeast;
#pragma unroll
            for (int gi = 0; gi < G; ++gi) {
              vz[mt][x2][gi] = __half22float2(pr[gi]);
              smax[mt][x2] = fmaxf(smax[mt][x2], vz[mt][x2][gi].x);
            }
          }
        uint32_t pf[NT][G][2][4];  // the weights times the values' scales, fp16 parts hi and lo, [8-key block]
        const auto weigh = [&](auto all) {
          constexpr bool kAll = decltype(all)::value;  // every (key, row) pair counts
          uint32_t vis = 0;  // else: bit nt * 8 + mt * 4 + (key half) * 2 + row
          if constexpr (!kAll) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int q = nt * 8 + 2 * t + i;
                if (q >= rows) continue;
                const int ti = (row0 + q) / gq;
                const unsigned long long* anc = a.mask ? a.mask + 2LL * (r.row + ti) : nullptr;
                const int qp = a.positions ? max(__ldg(a.positions + r.row + ti), r.first) : r.first + ti;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  if (sees(a, r, ti, qp, anc, kb + k * 8 + g)) vis |= 1u << (nt * 8 + k * 2 + i);
              }
          }
          const auto on = [&](int nt, int mt, int i) { return kAll || (vis >> (nt * 8 + mt * 4 + i) & 1u); };
          // weights, in units of 2^ref; twice where the reference has to rise first
          float w[NT][2][4];
#pragma unroll 1
          for (int again = 0; again < 2; ++again) {
            bool high = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  w[nt][mt][i] = on(nt, mt, i) ? ex2(sc[nt][mt][i] - ref[nt][i & 1]) : 0.f;
                  high |= w[nt][mt][i] * smax[mt][i >> 1] > kTop;
                }
            if (again || !__any_sync(0xffffffffu, high)) break;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                float top = -INFINITY;
                bool up = false;
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                  for (int x2 = 0; x2 < 2; ++x2)
                    if (on(nt, mt, x2 * 2 + i)) {
                      top = fmaxf(top, sc[nt][mt][2 * x2 + i] + __log2f(smax[mt][x2]));
                      up |= w[nt][mt][2 * x2 + i] * smax[mt][x2] > kTop;
                    }
#pragma unroll
                for (int x2 = 4; x2 < 32; x2 <<= 1) {
                  top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x2));
                  up |= __shfl_xor_sync(0xffffffffu, static_cast<int>(up), x2) != 0;
                }
                if (up) {
                  const float now = top - 7.f, al = ref[nt][i] == -INFINITY ? 1.f : ex2(ref[nt][i] - now);
                  ref[nt][i] = now;
                  l[nt][i] *= al;
#pragma unroll
                  for (int gi = 0; gi < G; ++gi) oz[nt][gi][i] *= al;
#pragma unroll
                  for (int x2 = 0; x2 < DB; ++x2)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                      o[nt][x2][y][i] *= al;
                      o[nt][x2][y][2 + i] *= al;
                    }
                }
              }
          }
          // sums, and the second product's operand: 8-key block k = 2 mt + x2 holds nibble k of V's words,
          // odd ones four bits up
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float w0 = w[nt][k >> 1][(k & 1) * 2], w1 = w[nt][k >> 1][(k & 1) * 2 + 1];
              const bool on0 = on(nt, k >> 1, (k & 1) * 2), on1 = on(nt, k >> 1, (k & 1) * 2 + 1);
              l[nt][0] += w0;
              l[nt][1] += w1;
#pragma unroll
              for (int gi = 0; gi < G; ++gi) {
                const float2 sz = vz[k >> 1][k & 1][gi];
                const float s2 = k & 1 ? sz.x * 0.0625f : sz.x;
                // (what a pair does not see may be NaN: selected away, not multiplied)
                oz[nt][gi][0] = on0 ? fmaf(w0, sz.y, oz[nt][gi][0]) : oz[nt][gi][0];
                oz[nt][gi][1] = on1 ? fmaf(w1, sz.y, oz[nt][gi][1]) : oz[nt][gi][1];
                const float p0 = on0 ? w0 * s2 : 0.f, p1 = on1 ? w1 * s2 : 0.f;
                const uint32_t hi = pack_f16(p0, p1);
                const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&hi));
                pf[nt][gi][0][k] = movmatrix_t(hi);
                pf[nt][gi][1][k] = movmatrix_t(pack_f16(p0 - back.x, p1 - back.y));
              }
            }
        };
        if (full)
          weigh(std::true_type{});
        else
          weigh(std::false_type{});
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const uint4 vw = *reinterpret_cast<const uint4*>(blk + B::kV + ((kg * (D / 4) + db * 8 + g) * 4 + t) * 16);
          const uint32_t x[4] = {vw.x, vw.y, vw.z, vw.w};
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const uint32_t x0 = x[2 * y], x1 = x[2 * y + 1], y0 = x0 >> 8, y1 = x1 >> 8;
            const uint32_t a0[4] = {x0 & 0x000f000fu, x1 & 0x000f000fu, x0 & 0x00f000f0u, x1 & 0x00f000f0u};
            const uint32_t a1[4] = {y0 & 0x000f000fu, y1 & 0x000f000fu, y0 & 0x00f000f0u, y1 & 0x00f000f0u};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
              for (int part = 0; part < 2; ++part) {
                mma_f16_16816(o[nt][db][y], a0, &pf[nt][db * 32 / kPgGroup][part][0]);
                mma_f16_16816(o[nt][db][y], a1, &pf[nt][db * 32 / kPgGroup][part][2]);
              }
            }
          }
        }
      }
      __syncwarp();  // every lane has read the stage
    }
    // ---- the segment's end: the warps' parts, joined through the stage that each read last ----
    const bool has = done > done0;
    float* buf = reinterpret_cast<float*>(ring + ((done + ST - 1) % ST) * B::kBytes);
    if (has) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int x2 = 4; x2 < 32; x2 <<= 1) {
            l[nt][i] += __shfl_xor_sync(0xffffffffu, l[nt][i], x2);
#pragma unroll
            for (int gi = 0; gi < G; ++gi) oz[nt][gi][i] += __shfl_xor_sync(0xffffffffu, oz[nt][gi][i], x2);
          }
          const int row = nt * 8 + 2 * t + i;
          if (g == 0) s_ml[warp][row] = make_float2(ref[nt][i], l[nt][i]);
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            float4 x;
            const float z = oz[nt][db * 32 / kPgGroup][i];
            x.x = fmaf(o[nt][db][0][i], 16777216.f, z);
            x.y = fmaf(o[nt][db][0][2 + i], 16777216.f, z);
            x.z = fmaf(o[nt][db][1][i], 16777216.f, z);
            x.w = fmaf(o[nt][db][1][2 + i], 16777216.f, z);
            // (16-byte chunks permuted by row so that a warp's store meets each bank once)
            *reinterpret_cast<float4*>(buf + row * D + (((db * 8 + g) ^ (2 * t)) << 2)) = x;
          }
        }
      }
    }
    if (lane == 0) s_has[warp] = has ? (done + ST - 1) % ST + 1 : 0;
    __syncthreads();
    const bool whole = pg0 == 0 && pg1 == r.pages;
    int c0 = 0, c1 = 0;  // CTAs that share the item
    if (!whole) {
      const long long T = p.total, Gd = gridDim.x;
      const int i0 = u - pg0, i1 = i0 + r.pages - 1;
      c0 = static_cast<int>(i0 * Gd / T);
      while ((c0 + 1) * T / Gd <= i0) ++c0;
      c1 = static_cast<int>(i1 * Gd / T);
      while ((c1 + 1) * T / Gd <= i1) ++c1;
    }
    const int slot = blockIdx.x * 2 + (pg0 == 0 ? 1 : 0);
    const auto finish = [&](int row, int c4, float M, float L, float4 x) {
      const float inv = L > 0.f ? 1.f / L : L == 0.f ? 0.f : L;  // (a NaN stays one)
      const float y[4] = {x.x * inv, x.y * inv, x.z * inv, x.w * inv};
      const int qr = row0 + row;
      const long long tok = r.row + qr / gq;
      const int head = h * gq + qr % gq;
      const long long at = tok * a.os + static_cast<long long>(head) * D + c4 * 4;
      if (a.is_half)
        store_vec<__half, 4>(static_cast<__half*>(a.out) + at, y);
      else
        store_vec<__nv_bfloat16, 4>(static_cast<__nv_bfloat16*>(a.out) + at, y);
      if (c4 == 0 && a.lse) a.lse[tok * a.hq + head] = (M + log2f(L)) * 0.6931471805599453f;
    };
    for (int x = tid; x < rows * (D / 4); x += W * 32) {
      const int row = x / (D / 4), c4 = x % (D / 4);
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int wi = 0; wi < W; ++wi)
        if (s_has[wi]) M = fmaxf(M, s_ml[wi][row].x);
      const float mb = M == -INFINITY ? 0.f : M;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int wi = 0; wi < W; ++wi) {
        const int st = s_has[wi];
        if (!st) continue;
        const float2 ml = s_ml[wi][row];
        const float fw = ex2(ml.x - mb);
        const float4 y = *reinterpret_cast<const float4*>(ring_all + (wi * ST + st - 1) * B::kBytes + (row * D + ((c4 ^ (2 * ((row >> 1) & 3))) << 2)) * 4);
        L = fmaf(fw, ml.y, L);
        sum.x = fmaf(fw, y.x, sum.x);
        sum.y = fmaf(fw, y.y, sum.y);
        sum.z = fmaf(fw, y.z, sum.z);
        sum.w = fmaf(fw, y.w, sum.w);
      }
      if (whole) {
        finish(row, c4, M, L, sum);
      } else {
        __stcg(reinterpret_cast<float4*>(p.part_o + (static_cast<long long>(slot) * R + row) * D) + c4, sum);
        if (c4 == 0) __stcg(p.part_ml + slot * R + row, make_float2(M, L));
      }
    }
    fence_async_smem();  // the parts in the stages, before copies write over them
    __syncthreads();
    if (!whole) {
      if (tid == 0) {
        s_last = atom_add_acq_rel_gpu(&p.counters[c0], 1) == c1 - c0;
        if (s_last) atomicExch(&p.counters[c0], 0);
      }
      __syncthreads();
      if (s_last) {
        for (int x = tid; x < rows * (D / 4); x += W * 32) {
          const int row = x / (D / 4), c4 = x % (D / 4);
          float M = -INFINITY, L = 0.f;
#pragma unroll 8
          for (int c = c0; c <= c1; ++c) M = fmaxf(M, __ldcg(p.part_ml + (c * 2 + (c == c0)) * R + row).x);
          const float mb = M == -INFINITY ? 0.f : M;
          float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int c = c0; c <= c1; ++c) {
            const long long sl = c * 2 + (c == c0);
            const float2 ml = __ldcg(p.part_ml + sl * R + row);
            const float4 y = __ldcg(reinterpret_cast<const float4*>(p.part_o + (sl * R + row) * D) + c4);
            const float fw = ex2(ml.x - mb);
            L = fmaf(fw, ml.y, L);
            sum.x = fmaf(fw, y.x, sum.x);
            sum.y = fmaf(fw, y.y, sum.y);
            sum.z = fmaf(fw, y.z, sum.z);
            sum.w = fmaf(fw, y.w, sum.w);
          }
          finish(row, c4, M, L, sum);
        }
      }
    }
    u = seg_end;
  }
  // after a wait gave up: the copies in flight land before the CTA ends
  if (!ok)
    for (int k = max(0, issued - ST); k < issued; ++k) mbar_drain(&bars[warp][k % ST], (k / ST) & 1);
}

template <int D, int NT>
cudaError_t pa_launch(const PaParams& p, int grid, cudaStream_t s) {
  paged_attn_kernel<D, NT><<<grid, PaShape<D, NT>::kWarps * 32, PaShape<D, NT>::kSmem, s>>>(p);
  return cudaGetLastError();
}
template <int D, int NT>
cudaError_t pa_prepare() {
  return cudaFuncSetAttribute(paged_attn_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              static_cast<int>(PaShape<D, NT>::kSmem));
}

}  // namespace

size_t pa_partial_rows(int sms) { return static_cast<size_t>(sms) * 2 * 16; }

cudaError_t pa_prepare_all() {
  cudaError_t e = pa_prepare<64, 1>();
  if (e == cudaSuccess) e = pa_prepare<64, 2>();
  if (e == cudaSuccess) e = pa_prepare<128, 1>();
  if (e == cudaSuccess) e = pa_prepare<128, 2>();
  return e;
}

cudaError_t launch_paged_attention(const tss_paged* h, const PgAttnParams& a, cudaStream_t s, bool* too_large) {
  *too_large = false;
  PaParams p{};
  p.a = a;
  p.part_o = h->part_o;
  p.part_ml = h->part_ml;
  p.counters = h->counters;
  const int gq = h->hq / h->hk;
  int most = 0;
  for (int i = 0; i < a.batch.n_req; ++i) most = a.batch.r[i].n * gq > most ? a.batch.r[i].n * gq : most;
  const int R = most <= 8 ? 8 : 16;
  long long at = 0;
  for (int i = 0; i < a.batch.n_req; ++i) {
    const PgReq& q = a.batch.r[i];
    if (q.n == 0) continue;
    PaReq& r = p.r[p.n_req++];
    r = PaReq{q.seq, q.first, q.n, q.row, 0, 0, 0, static_cast<int>(at)};
    const int end = (q.first + q.n + kPgTokens - 1) / kPgTokens;
    if (a.window) {
      r.lo = (q.first - a.window + 1 > 0 ? q.first - a.window + 1 : 0) / kPgTokens;
      const int sinks = a.sinks < q.first + q.n ? a.sinks : q.first + q.n;
      r.sink = (sinks + kPgTokens - 1) / kPgTokens;
      if (r.sink > r.lo) r.sink = r.lo;
    }
    r.pages = r.sink + end - r.lo;
    at += static_cast<long long>(r.pages) * h->hk * ((q.n * gq + R - 1) / R);
    if (at > 0x3fffffff) {
      *too_large = true;
      return cudaSuccess;
    }
  }
  p.total = static_cast<int>(at);
  const int grid = p.total < h->sms ? p.total : h->sms;
  if (h->d == 64) return R == 8 ? pa_launch<64, 1>(p, grid, s) : pa_launch<64, 2>(p, grid, s);
  return R == 8 ? pa_launch<128, 1>(p, grid, s) : pa_launch<128, 2>(p, grid, s);
}

}  // namespace tss
