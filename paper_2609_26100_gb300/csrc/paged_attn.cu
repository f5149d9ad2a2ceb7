// Attention of draft blocks over the paged 4-bit cache, on warp-level tensor cores.
//
//   score_tr = scale q_r . k_t,  k_t = s_t c_t + z_t per 64 dims   (row r, token t)
//   o_r = sum_t p_tr v_t / sum_t p_tr,  p_tr = 2^(log2e score_tr - ref_r),  v_t = s'_t c'_t + z'_t
//
// K's codes go to the tensor cores as they are: a nibble in the low bits of an fp16 lane is the subnormal
// number c 2^-24 (c 2^-20 four bits further up), so a 32-bit word becomes four operand registers with four
// ANDs and a shift, exactly; the factor 16 of every second pair is taken out of the other operand.  Scales
// and minima join in fp32: s_t multiplies the sum over a group's dims, z_t the sum of the query's; on the
// value side s'_t goes into the weight, which enters as two fp16 parts (hi and the rest, 22 bits) or, in blocks of more than
// 8 rows with bf16 outputs, as one (11 bits): beside bf16's own rounding errors, of 8 bits, it makes those of an output 0.8 %
// larger (of 2000, 9000 or 32768 keys alike), which the second part would buy back for an eighth of the time (64 samples over 32768 keys
// 202 -> 225 us); fp16's would be doubled.  The rest of the value is summed by itself, in fp32.  V's codes enter centred,
// v = s' (c' - 7.5) + (z' + 7.5 s'), one more operation a register, 2 to 5 % of the time: sums of terms of one sign drift (`centre`),
// and a rounded weight's error is multiplied by what it weighs: by codes as they are, whose mean square is six times that of
// centred ones, where the output is a mean over many keys and small.  Queries are scaled by a power of two to fill fp16's range, exact
// down to 2^-35 of a row's largest.
//
// Tokens take the MMA's 16-row side (S^T = K Q^T, O^T = V^T P^T): a block of 8 query rows (N) fills it,
// where the usual orientation would pad 1 .. 8 rows to 16.  P^T's operand layout is the transpose of S^T's
// accumulator: one movmatrix per 8 x 8.
//
// ref_r is raised only when some p s' passes 2^15 (fp16's end), to where the largest is between 2^6 and 2^7, so most tiles
// need no reduction over tokens.  In terms of p s' rather than p, it keeps the weights in fp16's range
// whatever the values' scales.  Each group of 64 dims has a reference of its own (as a power of two beside the first
// group's), since one group's scales may be a millionth of the other's: under the other's reference its weights would be
// fp16 subnormals, and its dims off by 1e-2.
//
// Work split.  A unit is a page (or half of one, for short launches) of one item: a request's row tile and KV
// head.  CTAs of four warps, three to an SM (two with 16 rows), take runs of units; a run's units go round its
// warps, each with its own ring of bulk copies.  Several small CTAs rather than one: while one ends an item the
// others stream.  At an item's end the warps' parts are joined in shared memory; items that several CTAs share
// leave partials, which the last CTA to arrive joins in CTA order (results do not depend on timing).
//
// Bound: up to 8 rows, instruction issue and HBM together: 4 x 65536 keys, 32 heads, 1 row in 234 us, 5.2 TB/s (over a third of
// the 608 instructions that a warp spends on 32 keys and 8 rows take codes apart; 12 warps an SM, as many as 168 registers
// allow, issue in 58 % of the cycles); beyond, neither: eight warps an SM (249 registers) do not hide the steps from load to
// MMA, 16 x 16384 keys, 9 rows in 332 us.  One token over 1024 keys takes 9.4 us: launch, table, page, two joins.
#include <type_traits>

#include "paged_attn.cuh"

namespace tss {
namespace {

__device__ __forceinline__ uint32_t movmatrix_t(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// d += a b and d = a b, fp16 in, fp32 out.  (Not volatile: the compiler may place them among the integer work.)
__device__ __forceinline__ void mma_next(float* d, const uint32_t* a, const uint32_t* b) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ void mma_first(float* d, const uint32_t* a, const uint32_t* b) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]), "f"(0.f));
}

// A ring stage holds a page's block (or half of each of its parts).  W: warps of a CTA, 4, or 1 for many short items.
template <int D, int NT, int W>
struct PaShape {
  static constexpr int kRows = 8 * NT;
  static constexpr int kWarps = W;
  static constexpr int kCtas = W == 1 ? (NT == 1 ? 11 : 8) : NT == 1 ? 3 : 2;  // resident on an SM
  static constexpr int kStages = NT == 1 || W == 1 ? 2 : 3;
  static constexpr size_t kSmem = kWarps * kStages * PgBlock<D>::kBytes;
};

// Whether row i (position qp, mask words anc or null) of request r sees key j.
__device__ __forceinline__ bool sees(const PgAttnArgs& a, const PaReq& r, int i, int qp, const unsigned long long* anc, int j) {
  if (j >= r.first + r.n) return false;
  int kp = j;
  if (j >= r.first) {
    const int x = j - r.first;
    if (anc ? !(__ldcg(anc + (x >> 6)) >> (x & 63) & 1ull) : x > i) return false;
    if (a.positions) kp = max(__ldcg(a.positions + r.row + x), r.first);
  }
  return !a.window || qp - kp < a.window || j < a.sinks;
}

// TWO: weights of two fp16 parts.  SH: a pass of the attention of sequences that share keys.
template <int D, int NT, bool TWO, bool SH, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, PaShape<D, NT, WARPS>::kCtas)
    paged_attn_kernel(const __grid_constant__ typename PaParamsOf<SH>::type p) {
  using B = PgBlock<D>;
  using S = PaShape<D, NT, WARPS>;
  constexpr int G = B::kGroups, W = S::kWarps, ST = S::kStages, R = S::kRows, DB = D / 32;
  extern __shared__ __align__(128) uint8_t pa_dyn[];
  __shared__ uint64_t bars[W][ST];
  __shared__ int s_off[kPgMaxReq], s_qp[W][R];  // s_qp: positions of the rows that the warp works on
  __shared__ float2 s_ml[W][R];
  __shared__ int s_has[W], abort_s, s_last;  // s_has: the stage of a warp's part, plus one; 0 without
  __shared__ __align__(16) float s_x[W][D];  // parts of rows that several warps gather from other CTAs' partials
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  uint8_t* ring = pa_dyn + warp * (ST * B::kBytes);
  const PgAttnArgs& a = p.a;
  const int gq = a.hq / a.hk, halves = p.halves, unit = 32 * halves;  // tokens of a unit
  for (int i = tid; i < p.n_req; i += W * 32) s_off[i] = p.r[i].off;
  if (lane == 0)
    for (int i = 0; i < ST; ++i) mbar_init(&bars[warp][i], 1);
  if (tid == 0) abort_s = 0;
  fence_mbar_init();
  // the CTA's run of units [u0, u1)
  int u0, u1, first_cta, splits;
  cta_run(p, &u0, &u1, &first_cta, &splits);
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
  // Lane l: entry of the table for unit k0 + l (-1 past the end), and its KV head and half of the page.
  const auto place_of = [&](int k0, int* part) -> long long {
    if (k0 + lane >= mine) return -1;
    const int u = u0 + warp + (k0 + lane) * W, b = request_of(u), v = u - s_off[b];
    const PaReq& r = p.r[b];
    const int item = v / r.units, x = v - item * r.units;
    const int at = x < r.sink ? x : x - r.sink + r.lo;
    *part = item % a.hk * 2 + (halves == 1 ? at & 1 : 0);
    return static_cast<long long>(r.seq) * a.max_pages + (halves == 1 ? at >> 1 : at);
  };
  // Half block in the pool; -1 where the table names no page, -2 past the end.
  const auto block_at = [&](long long place, int part) -> int {
    if (place < 0) return -2;
    const int page = __ldcg(a.table + place);
    if (page < 0 || page >= a.n_pages) {
      report(a.status, kStatusCheck);
      return -1;
    }
    return page * a.hk * 2 + part;  // (below 2^31: the host checks)
  };
  int part = 0;
  const long long place = place_of(0, &part);
  // Nothing before this reads or writes what another kernel may; tables, masks and positions are not read through the
  // read-only path, since the kernel that writes them may still run while this one begins.
  if constexpr (SH) {
    if (!p.early) griddep_wait();  // (what this reads before that was complete when the pass before it began)
  } else {
    griddep_wait();
  }
  griddep_launch();
  int ids = block_at(place, part), ids_next = -2;
  int issued = 0, issue_at = 0;  // units asked for, the stage of the next
  uint32_t no_page = 0;  // bit s: stage s's unit has no page
  // a unit's copies: lane 0 K codes, 1 V codes, 2 K parameters, 3 V parameters
  const int piece_half = (lane < 2 ? B::kCodes : B::kParams) / 2, piece = piece_half * halves;
  const int piece_at = lane < 2 ? lane * B::kCodes : B::kKParams + (lane - 2) * B::kParams;
  const bool withheld = p.withhold && blockIdx.x == 0 && warp == 0;
  const auto issue = [&]() {  // the warp's next unit into stage issued % ST
    if (issued >= mine) return;
    if ((issued & 31) == 0) {
      if (issued > 0) ids = ids_next;
      if (issued + 32 < mine) {
        const long long next = place_of(issued + 32, &part);
        ids_next = block_at(next, part);
      }
    }
    const int blk = __shfl_sync(0xffffffffu, ids, issued & 31), s = issue_at;
    issue_at = s + 1 == ST ? 0 : s + 1;
    if (blk < 0) {
      no_page |= 1u << s;
      if (lane == 0) mbar_arrive(&bars[warp][s]);
    } else {
      no_page &= ~(1u << s);
      uint64_t* bar = &bars[warp][s];
      if (lane == 0) mbar_arrive_expect_tx(bar, B::kBytes / 2 * halves);
      __syncwarp();
      if (lane < 4 && !withheld)
        bulk_load(ring + s * B::kBytes + piece_at, a.pool + static_cast<long long>(blk >> 1) * B::kBytes + piece_at + (blk & 1) * piece_half, piece,
                  bar);
    }
    ++issued;
  };
  // All stages but one: the last is asked for at the first unit, so that first pages and Q do not queue behind second ones
  // (eight requests of 4000 tokens, 32 heads, 44.8 -> 43.3 us).
#pragma unroll
  for (int i = 0; i < ST - 1; ++i) issue();

  int done = 0, stage = 0;  // the warp's units so far, the stage of the next
  uint32_t parity = 0;
  bool ok = true;
  for (int u = u0; u < u1;) {
    // ---- a segment: this CTA's units [x0, x1) of an item ----
    const int b = request_of(u);
    const PaReq& r = p.r[b];
    const int v = u - r.off, item = v / r.units, x0 = v - item * r.units;
    const int seg_end = min(u1, u - x0 + r.units), x1 = x0 + seg_end - u;
    const int h = item % a.hk, row0 = item / a.hk * R, rows = min(R, r.n * gq - row0);
    // Q: thread (g, t) holds row g's dims 64 gi + 16 t .. + 15 as the operand of 4 k-steps a group: pairs
    // (0, 4), (1, 5) and (2, 6), (3, 7) of each 8 dims, odd ones / 16 (their codes stand four bits up)
    uint32_t qf[NT][G][2][4];
    float2 f2[NT], ref2[NT], l2[NT];  // (of rows 2t and 2t + 1; the reference negated)
    float zq[NT][G][2], oz[NT][G][2], o[NT][DB][2][4];
    float2 gx[NT];  // G == 2: what turns weights under the first group's reference into those under the second's
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
      const float up = query_scale(big);
      const float mul = a.scale_log2 * 16777216.f / up;
      float sum[G];
#pragma unroll
      for (int gi = 0; gi < G; ++gi) {
        sum[gi] = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[gi] += x[gi][i];
        sum[gi] += __shfl_xor_sync(0xffffffffu, sum[gi], 1);
        sum[gi] += __shfl_xor_sync(0xffffffffu, sum[gi], 2);
        sum[gi] *= up * 5.9604645e-8f;  // (f times this is scale_log2)
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float m = i & 1 ? up * 0.0625f : up;
            qf[nt][gi][w][i] = pack_f16(x[gi][8 * w + i] * m, x[gi][8 * w + i + 4] * m);
          }
      }
      // the accumulators' rows of a thread are 2t and 2t + 1
      f2[nt] = make_float2(__shfl_sync(0xffffffffu, mul, 8 * t), __shfl_sync(0xffffffffu, mul, 8 * t + 4));
      ref2[nt] = make_float2(INFINITY, INFINITY);
      l2[nt] = make_float2(0.f, 0.f);
      gx[nt] = make_float2(1.f, 1.f);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
          zq[nt][gi][i] = __shfl_sync(0xffffffffu, sum[gi], 8 * t + 4 * i);
          oz[nt][gi][i] = 0.f;
        }
#pragma unroll
      for (int x2 = 0; x2 < DB; ++x2)
#pragma unroll
        for (int i = 0; i < 8; ++i) o[nt][x2][i >> 2][i & 3] = 0.f;
    }
    if (a.window) {  // the last position among the tile's rows
      if (lane < rows) {
        pmax = row_position(p, r, (row0 + lane) / gq);
        if constexpr (SH) s_qp[warp][lane] = pmax;
      }
#pragma unroll
      for (int x2 = 16; x2 > 0; x2 >>= 1) pmax = max(pmax, __shfl_xor_sync(0xffffffffu, pmax, x2));
      if constexpr (SH) __syncwarp();  // (the positions, before other lanes read them: shuffles order no memory)
    }
    int all0, all1, all2;
    units_in_sight(a, r, unit, pmax, &all0, &all1, &all2);
    const int done0 = done;
    // (After a wait gave up the warp asks for nothing more and waits for nothing, in this segment and those after it: an
    // arrival at a stage whose copy is still on its way would be one too many for its barrier.)
    for (int x = u0 + warp + done * W - u + x0; ok && x < x1; x += W) {
      issue();  // into the stage of the unit before, if any (every lane has read it: the last loop's end)
      const int s = stage;
      if (!__all_sync(0xffffffffu, mbar_try_wait(&bars[warp][s], parity))) {
        ok = __all_sync(0xffffffffu, ok && mbar_wait(&bars[warp][s], parity, abort, a.status));
        if (!ok) break;
      }
      ++done;
      stage = s + 1 == ST ? 0 : s + 1;
      parity ^= stage == 0;
      const bool full = no_page == 0 && (x < all0 || (x >= all1 && x < all2));
      if (no_page >> s & 1u) continue;
#pragma unroll 1
      for (int kg = 0; kg < halves; ++kg) {
        const uint8_t* blk = ring + s * B::kBytes;
        const uint8_t *kcodes = blk + B::kK + kg * (B::kCodes / 2), *vcodes = blk + B::kV + kg * (B::kCodes / 2);
        const __half2* kparams = reinterpret_cast<const __half2*>(blk + B::kKParams) + kg * 32 * G;
        const __half2* vparams = reinterpret_cast<const __half2*>(blk + B::kVParams) + kg * 32 * G;
        float sc[NT][2][4];  // scores / f: [16-key tile][key g, rows 2t and 2t + 1; key g + 8, the same]
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
          float acc[NT][G][4];
          uint32_t kw[2][G][2];
#pragma unroll
          for (int x2 = 0; x2 < 2; ++x2) {
            const uint8_t* kp = kcodes + (mt * 16 + x2 * 8 + g) * (D / 2) + t * (D / 8);
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
                if (w == 0)
                  mma_first(acc[nt][gi], a0, &qf[nt][gi][w][0]);
                else
                  mma_next(acc[nt][gi], a0, &qf[nt][gi][w][0]);
                mma_next(acc[nt][gi], a1, &qf[nt][gi][w][2]);
              }
            }
          // scores from the codes' sums
#pragma unroll
          for (int x2 = 0; x2 < 2; ++x2) {
            const __half2* pr = kparams + (mt * 16 + x2 * 8 + g) * G;
            float2 sz[G];
#pragma unroll
            for (int gi = 0; gi < G; ++gi) sz[gi] = __half22float2(pr[gi]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                float c = sz[0].x * acc[nt][0][2 * x2 + i];
                if constexpr (G == 2) c = fmaf(sz[G - 1].x, acc[nt][G - 1][2 * x2 + i], c);
#pragma unroll
                for (int gi = 0; gi < G; ++gi) c = fmaf(sz[gi].y, zq[nt][gi][i], c);
                sc[nt][mt][2 * x2 + i] = c;
              }
          }
        }
        float2 vz[2][2][G];
        float smax[G];  // the largest scale among the thread's keys
#pragma unroll
        for (int gi = 0; gi < G; ++gi) smax[gi] = kLeast;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const __half2* pr = vparams + (k * 8 + g) * G;
#pragma unroll
          for (int gi = 0; gi < G; ++gi) {
            vz[k >> 1][k & 1][gi] = __half22float2(pr[gi]);
            vz[k >> 1][k & 1][gi].y = fmaf(vz[k >> 1][k & 1][gi].x, 7.5f, vz[k >> 1][k & 1][gi].y);  // (v = s' (c' - 7.5) + (z' + 7.5 s'))
            smax[gi] = fmaxf(smax[gi], vz[k >> 1][k & 1][gi].x);
          }
        }
        constexpr int kParts = TWO ? 2 : 1;
        uint32_t pf[NT][G][kParts][4];  // the weights times the values' scales in fp16 parts, [8-key block]
        const auto weigh = [&](auto all) {
          constexpr bool kAll = decltype(all)::value;  // every (key, row) pair counts
          uint32_t vis = 0;  // else: bit nt * 8 + mt * 4 + (key half) * 2 + row
          if constexpr (!kAll) {
            const int kb = (x < r.sink ? x : x - r.sink + r.lo) * unit + kg * 32;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int q = nt * 8 + 2 * t + i;
                if (q >= rows) continue;
                const int ti = (row0 + q) / gq;
                const unsigned long long* anc = a.mask ? a.mask + 2LL * (r.row + ti) : nullptr;
                int qp;
                if constexpr (SH)
                  qp = a.window ? s_qp[warp][q] : 0;  // (read only under a window)
                else
                  qp = row_position(p, r, ti);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  if (sees(a, r, ti, qp, anc, kb + k * 8 + g)) vis |= 1u << (nt * 8 + k * 2 + i);
              }
          }
          const auto on = [&](int nt, int mt, int i) { return kAll || (vis >> (nt * 8 + mt * 4 + i) & 1u); };
          // weights, in units of 2^ref; again where the reference has to rise first
          float w[NT][2][4];
          float wmax[G];  // the thread's largest, under each group's reference
          const auto weights = [&]() {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float2 m = make_float2(0.f, 0.f);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                float* sp = &sc[nt][k >> 1][(k & 1) * 2];
                float* wp = &w[nt][k >> 1][(k & 1) * 2];
                const float2 e = fma2(make_float2(sp[0], sp[1]), f2[nt], ref2[nt]);
                wp[0] = on(nt, k >> 1, (k & 1) * 2) ? ex2(e.x) : 0.f;
                wp[1] = on(nt, k >> 1, (k & 1) * 2 + 1) ? ex2(e.y) : 0.f;
                m = make_float2(fmaxf(m.x, wp[0]), fmaxf(m.y, wp[1]));
              }
              wmax[0] = nt ? fmaxf(wmax[0], fmaxf(m.x, m.y)) : fmaxf(m.x, m.y);
              if constexpr (G == 2) {
                const float x = fmaxf(m.x * gx[nt].x, m.y * gx[nt].y);
                wmax[G - 1] = nt ? fmaxf(wmax[G - 1], x) : x;
              }
            }
          };
          weights();
          // (the thread's largest weight and scale may be of different keys: then nothing rises below)
          bool over = false;
#pragma unroll
          for (int gi = 0; gi < G; ++gi) over |= wmax[gi] * smax[gi] > kTop;
          if (__any_sync(0xffffffffu, over)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                float& ref = i ? ref2[nt].y : ref2[nt].x;
                float& factor = i ? gx[nt].y : gx[nt].x;
                float top[G];
#pragma unroll
                for (int gi = 0; gi < G; ++gi) top[gi] = -INFINITY;
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                  for (int x2 = 0; x2 < 2; ++x2)
                    if (on(nt, mt, x2 * 2 + i)) {
#pragma unroll
                      for (int gi = 0; gi < G; ++gi)
                        top[gi] = fmaxf(top[gi], fmaf(sc[nt][mt][2 * x2 + i], i ? f2[nt].y : f2[nt].x, __log2f(fmaxf(vz[mt][x2][gi].x, kLeast))));
                    }
#pragma unroll
                for (int x2 = 4; x2 < 32; x2 <<= 1)
#pragma unroll
                  for (int gi = 0; gi < G; ++gi) top[gi] = fmaxf(top[gi], __shfl_xor_sync(0xffffffffu, top[gi], x2));
                // (negated, and whole numbers, so that the factor between the groups is a power of two; infinite until the row's
                // first keys, which set both)
                const float last = ref + static_cast<float>((__float_as_int(factor) >> 23) - 127);  // of the last group
                const bool up = top[0] + ref > 15.f, up_last = top[G - 1] + last > 15.f;
                if (up || up_last) {
                  const bool first = ref == INFINITY;
                  const float now = up ? floorf(7.f - top[0]) : ref, al = first ? 1.f : pow2(now - ref);
                  float al_last = al;
                  if constexpr (G == 2) {
                    const float now_last = up_last ? floorf(7.f - top[G - 1]) : last;
                    al_last = first ? 1.f : pow2(now_last - last);
                    factor = pow2(now_last - now);
                  }
                  ref = now;
                  (i ? l2[nt].y : l2[nt].x) *= al;
#pragma unroll
                  for (int gi = 0; gi < G; ++gi) oz[nt][gi][i] *= al;
#pragma unroll
                  for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                      o[nt][db][y][i] *= db * 32 / kPgGroup ? al_last : al;
                      o[nt][db][y][2 + i] *= db * 32 / kPgGroup ? al_last : al;
                    }
                }
              }
            weights();
          }
          // sums, and the second product's operand: 8-key block k = 2 mt + x2 holds nibble k of V's words,
          // odd ones four bits up
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float w0 = w[nt][k >> 1][(k & 1) * 2], w1 = w[nt][k >> 1][(k & 1) * 2 + 1];
              const bool on0 = on(nt, k >> 1, (k & 1) * 2), on1 = on(nt, k >> 1, (k & 1) * 2 + 1);
              l2[nt] = add2(l2[nt], make_float2(w0, w1));
              const float2 wx = G == 2 ? mul2(make_float2(w0, w1), gx[nt]) : make_float2(0.f, 0.f);
#pragma unroll
              for (int gi = 0; gi < G; ++gi) {
                const float2 sz = vz[k >> 1][k & 1][gi];
                // (what a pair does not see may be NaN: selected away, not multiplied)
                oz[nt][gi][0] = on0 ? fmaf(w0, sz.y, oz[nt][gi][0]) : oz[nt][gi][0];
                oz[nt][gi][1] = on1 ? fmaf(w1, sz.y, oz[nt][gi][1]) : oz[nt][gi][1];
                const float2 pw = mul2(gi ? wx : make_float2(w0, w1), make_float2(sz.x, sz.x));
                const float p0 = on0 ? pw.x : 0.f, p1 = on1 ? pw.y : 0.f;
                const uint32_t hi = pack_f16(p0, p1);
                pf[nt][gi][0][k] = movmatrix_t(hi);
                if constexpr (TWO) {
                  const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&hi));
                  const float2 rest = fma2(back, make_float2(-1.f, -1.f), make_float2(p0, p1));
                  pf[nt][gi][kParts - 1][k] = movmatrix_t(pack_f16(rest.x, rest.y));
                }
              }
            }
        };
        if (full)
          weigh(std::true_type{});
        else
          weigh(std::false_type{});
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const uint4 vw = *reinterpret_cast<const uint4*>(vcodes + ((db * 8 + g) * 4 + t) * 16);
          const uint32_t x[4] = {vw.x, vw.y, vw.z, vw.w};
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const uint32_t x0 = x[2 * y], x1 = x[2 * y + 1], y0 = x0 >> 8, y1 = x1 >> 8;
            uint32_t a0[4] = {x0 & 0x000f000fu, x1 & 0x000f000fu, x0 & 0x00f000f0u, x1 & 0x00f000f0u};
            uint32_t a1[4] = {y0 & 0x000f000fu, y1 & 0x000f000fu, y0 & 0x00f000f0u, y1 & 0x00f000f0u};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              a0[i] = centre(a0[i], i >= 2);
              a1[i] = centre(a1[i], i >= 2);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const uint32_t(&w)[kParts][4] = pf[nt][db * 32 / kPgGroup];
#pragma unroll
              for (int part = 0; part < kParts; ++part) {
                mma_next(o[nt][db][y], a0, &w[part][0]);
                mma_next(o[nt][db][y], a1, &w[part][2]);
              }
            }
          }
        }
      }
      __syncwarp();
    }
    // ---- the segment's end: the warps' parts, joined through the stage that each read last ----
    const int last = stage == 0 ? ST - 1 : stage - 1;
    if (lane == 0) s_has[warp] = done > done0 ? last + 1 : 0;
    if (done > done0) {
      float* buf = reinterpret_cast<float*>(ring + last * B::kBytes);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int x2 = 4; x2 < 32; x2 <<= 1) {
            float& l = i ? l2[nt].y : l2[nt].x;
            l += __shfl_xor_sync(0xffffffffu, l, x2);
#pragma unroll
            for (int gi = 0; gi < G; ++gi) oz[nt][gi][i] += __shfl_xor_sync(0xffffffffu, oz[nt][gi][i], x2);
          }
          const int row = nt * 8 + 2 * t + i;
          if (g == 0) s_ml[warp][row] = i ? make_float2(-ref2[nt].y, l2[nt].y) : make_float2(-ref2[nt].x, l2[nt].x);
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            float4 x;
            const float z = oz[nt][db * 32 / kPgGroup][i];
            // (2^9 over the group's factor, a power of two)
            constexpr uint32_t kUp = 9;
            const float m = db * 32 / kPgGroup ? __uint_as_float(((kUp + 254u) << 23) - __float_as_uint(i ? gx[nt].y : gx[nt].x))
                                               : static_cast<float>(1 << kUp);
            x.x = fmaf(o[nt][db][0][i], m, z);
            x.y = fmaf(o[nt][db][0][2 + i], m, z);
            x.z = fmaf(o[nt][db][1][i], m, z);
            x.w = fmaf(o[nt][db][1][2 + i], m, z);
            // (16-byte chunks permuted by row so that a warp's store meets each bank once)
            *reinterpret_cast<float4*>(buf + row * D + (((db * 8 + g) ^ (2 * t)) << 2)) = x;
          }
        }
      }
      fence_async_smem();  // (the next segment's first copy goes to this stage: stores before the async proxy's)
    }
    __syncthreads();
    const bool whole = x0 == 0 && x1 == r.units;
    if (whole) wait_for_shared(p);  // (else the join does)
    int c0 = first_cta, c1 = first_cta + splits - 1;  // CTAs that share the item
    if (!whole && !p.aligned) {
      c0 = cta_of_unit(p, b, u - x0);
      c1 = cta_of_unit(p, b, u - x0 + r.units - 1);
    }
    // a CTA's two partials: of the item that it begins, and of the one that it ends or runs through
    const int slot = blockIdx.x * 2 + (x0 == 0 ? 1 : 0);
    const auto finish = [&](int row, int c4, float M, float L, float4 x) { finish_row<D>(p, r, h, row0 + row, c4, M, L, x); };
    // the parts of (row, 4 dims), with the rows' references and sums
    const auto joined = [&](int row, int c4, float2* ml, float4* sum) {
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int wi = 0; wi < W; ++wi)
        if (s_has[wi]) M = fmaxf(M, s_ml[wi][row].x);
      const float mb = M == -INFINITY ? 0.f : M;
      *sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int wi = 0; wi < W; ++wi) {
        if (!s_has[wi]) continue;
        const float2 x = s_ml[wi][row];
        const float fw = ex2(x.x - mb);
        const float* buf = reinterpret_cast<const float*>(pa_dyn + (wi * ST + s_has[wi] - 1) * B::kBytes);
        const float4 y = *reinterpret_cast<const float4*>(buf + row * D + ((c4 ^ (2 * ((row >> 1) & 3))) << 2));
        L = fmaf(fw, x.y, L);
        sum->x = fmaf(fw, y.x, sum->x);
        sum->y = fmaf(fw, y.y, sum->y);
        sum->z = fmaf(fw, y.z, sum->z);
        sum->w = fmaf(fw, y.w, sum->w);
      }
      *ml = make_float2(M, L);
    };
    for (int x = tid; x < rows * (D / 4); x += W * 32) {
      const int row = x / (D / 4), c4 = x % (D / 4);
      float2 ml;
      float4 sum;
      joined(row, c4, &ml, &sum);
      if (whole) {
        finish(row, c4, ml.x, ml.y, sum);
      } else {
        __stcg(reinterpret_cast<float4*>(p.part_o + (static_cast<long long>(slot) * R + row) * D) + c4, sum);
        if (c4 == 0) __stcg(p.part_ml + slot * R + row, ml);
      }
    }
    __syncthreads();
    if (!whole) {
      if (tid == 0) {
        s_last = atom_add_acq_rel_gpu(&p.counters[c0], 1) == c1 - c0;
        if (s_last) atomicExch(&p.counters[c0], 0);
      }
      __syncthreads();
      if (s_last) {
        // Few rows: several warps take a row, each some of its partials.
        const int per_row = W == 1 ? 1 : rows == 1 ? W : rows == 2 ? W / 2 : 1, slice = warp % per_row;
        for (int row = warp / per_row; row < rows; row += W / per_row) {
          float M, L;
          float4 sum;
          gather_partials<D>(p, R, c0, c1, row, slice, per_row, &M, &L, &sum);
          if (per_row == 1) {
            wait_for_shared(p);
            if (lane < D / 4) finish(row, lane, M, L, sum);
          } else {
            const int at = slice * rows + row;  // (at most W)
            if (lane == 0) s_ml[at][0] = make_float2(M, L);
            if (lane < D / 4) reinterpret_cast<float4*>(s_x[at])[lane] = sum;
          }
        }
        __syncthreads();
        if (per_row > 1) {
          wait_for_shared(p);
          for (int x = tid; x < rows * (D / 4); x += W * 32) {
            const int row = x / (D / 4), c4 = x % (D / 4);
            float M = -INFINITY, L = 0.f;
            for (int k = 0; k < per_row; ++k) M = fmaxf(M, s_ml[k * rows + row][0].x);
            const float mb = M == -INFINITY ? 0.f : M;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int k = 0; k < per_row; ++k) {
              const float2 ml = s_ml[k * rows + row][0];
              const float4 y = reinterpret_cast<const float4*>(s_x[k * rows + row])[c4];
              const float fw = ex2(ml.x - mb);
              L = fmaf(fw, ml.y, L);
              sum.x = fmaf(fw, y.x, sum.x);
              sum.y = fmaf(fw, y.y, sum.y);
              sum.z = fmaf(fw, y.z, sum.z);
              sum.w = fmaf(fw, y.w, sum.w);
            }
            finish(row, c4, M, L, sum);
          }
          __syncthreads();
        }
      }
    }
    u = seg_end;
  }
  wait_for_shared(p);  // (a CTA without work too: the kernel ends no earlier than the one before it)
  // after a wait gave up: the copies in flight land before the CTA ends
  if (!ok && !withheld)
    for (int k = max(0, issued - ST); k < issued; ++k) mbar_drain(&bars[warp][k % ST], (k / ST) & 1);
}

template <int D, int NT, bool TWO>
cudaError_t pa_launch(PaShared& p, bool shared, int sms, cudaStream_t s) {
  using S = PaShape<D, NT, 4>;
  // A run of a unit for each warp at least.  Leads of 0 / 3 / 6 / 10 / 16 pages, us: six requests of 60 to 30000
  // tokens 180 / 100 / 66 / 53 / 50, eight of 512 to 4096 45 / 40 / 38 / 37 / 38, equal ones alike at any.
  const int grid = pa_cut(p, sms * S::kCtas, S::kWarps, 8, 10 * (3 - p.halves));
  const dim3 g(grid), b(S::kWarps * 32);
  return shared ? launch_k(paged_attn_kernel<D, NT, TWO, true, 4>, g, b, S::kSmem, s, true, p)
                : launch_k(paged_attn_kernel<D, NT, TWO, false, 4>, g, b, S::kSmem, s, true, static_cast<PaParams&>(p));
}
// A warp for every item.
template <int D, int NT, bool TWO>
cudaError_t pa_launch_items(PaShared& p, cudaStream_t s) {
  using S = PaShape<D, NT, 1>;
  return launch_k(paged_attn_kernel<D, NT, TWO, true, 1>, dim3(pa_each(p)), dim3(32), S::kSmem, s, true, p);
}
template <int D, int NT, bool TWO>
cudaError_t pa_prepare() {
  const auto allow = [](auto kernel, size_t bytes) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes)); };
  cudaError_t e = allow(paged_attn_kernel<D, NT, TWO, false, 4>, PaShape<D, NT, 4>::kSmem);
  if (e == cudaSuccess) e = allow(paged_attn_kernel<D, NT, TWO, true, 4>, PaShape<D, NT, 4>::kSmem);
  if (e == cudaSuccess) e = allow(paged_attn_kernel<D, NT, TWO, true, 1>, PaShape<D, NT, 1>::kSmem);
  return e;
}

// What a pass writes its partial results to, and whether it waits for the pass before it only where it joins.
struct PaWork {
  float* part_o;
  float2* part_ml;
  int* counters;
  int early;
};

// The launches of a pass: blocks of more than `limit` query rows of a KV head go to the tcgen05 kernel (head_dim 128), the others
// to the one above.
cudaError_t pa_pass(tss_paged* h, const PgAttnArgs& a, const PaTask* tasks, int n_tasks, const int2* mem, int limit, const PaWork& work, int withhold,
                    bool shared, cudaStream_t s, bool* too_large) {
  PaTask few[kPgMaxReq], many[kPgMaxReq];
  int n_few = 0, n_many = 0, most = 0;
  for (int i = 0; i < n_tasks; ++i) {
    const PaTask& t = tasks[i];
    if (t.rows == 0) continue;
    if (h->d == 128 && t.rows > limit) {
      many[n_many++] = t;
    } else {
      few[n_few++] = t;
      most = t.rows > most ? t.rows : most;
    }
  }
  PaShared p, narrow;
  const auto begin = [&](PaShared& x) {
    x.a = a;
    x.part_o = work.part_o;
    x.part_ml = work.part_ml;
    x.counters = work.counters;
    x.early = work.early;
    x.withhold = withhold;
    if (mem)
      for (int i = 0; i < kPgMaxReq; ++i) x.mem[i] = mem[i];
  };
  if (n_many) {
    begin(p);
    if (!pa_plan(p, many, n_many, kPaTcTile, 2)) {
      *too_large = true;
      return cudaSuccess;
    }
  }
  if (n_few) {
    begin(narrow);
    const int R = most <= 8 ? 8 : 16;
    // Units of a page; of half a page where that leaves the warps less than three pages each (a warp takes
    // about 2 us for a page, so a short launch is as long as its longest warp).
    bool fits = pa_plan(narrow, few, n_few, R, 2);
    // Own keys beside a shared prefix are few as a rule and their items many: a warp for each, where the SMs' warps take that
    // sooner than the four of a CTA, which share an item and join (about 4 us an item, and 2 a page of a warp).
    bool each = false;
    if (fits && shared && a.own && narrow.n_req) {
      const auto items = [&](int i) { return ((i + 1 < narrow.n_req ? narrow.r[i + 1].off : narrow.total) - narrow.r[i].off) / narrow.r[i].units; };
      int n = 0, longest = 0;
      for (int i = 0; i < narrow.n_req; ++i) {
        n += items(i);
        longest = narrow.r[i].units > longest ? narrow.r[i].units : longest;
      }
      const double one = h->sms * (R == 8 ? 11. : 8.), four = h->sms * (R == 8 ? 3. : 2.);
      const double mean = static_cast<double>(narrow.total) / n;
      each = (n > one ? n / one * (4 + 2 * mean) : 4 + 2 * longest) < (n > four ? n / four : 1) * (5 + mean / 2);
    }
    if (fits && !each && narrow.total < 3LL * h->sms * (R == 8 ? 12 : 8)) fits = pa_plan(narrow, few, n_few, R, 1);
    if (!fits) {
      *too_large = true;
      return cudaSuccess;
    }
    const auto run = [&](auto dim) {
      constexpr int D = decltype(dim)::value;
      if (each) {
        if (R == 8) return pa_launch_items<D, 1, true>(narrow, s);
        return a.is_half ? pa_launch_items<D, 2, true>(narrow, s) : pa_launch_items<D, 2, false>(narrow, s);
      }
      if (R == 8) return pa_launch<D, 1, true>(narrow, shared, h->sms, s);
      return a.is_half ? pa_launch<D, 2, true>(narrow, shared, h->sms, s) : pa_launch<D, 2, false>(narrow, shared, h->sms, s);
    };
    if (narrow.n_req) {
      const cudaError_t e = h->d == 64 ? run(std::integral_constant<int, 64>{}) : run(std::integral_constant<int, 128>{});
      if (e != cudaSuccess) return e;
      p.early = 0;  // (behind the launch above now, whose workspace it shares)
    }
  }
  return n_many && p.n_req ? launch_paged_attention_tc(p, shared, h->sms, s) : cudaSuccess;
}

}  // namespace

// (two partials of 8 rows for three CTAs of an SM, of 16 for two, of 128 for one of the tcgen05 kernel)
size_t pa_partial_rows(int sms, int head_dim) { return static_cast<size_t>(sms) * 2 * (head_dim == 128 ? 128 : 32); }
int pa_counters(int sms) { return sms * 3; }

cudaError_t pa_prepare_all() {
  cudaError_t e = pa_prepare<64, 1, true>();
  if (e == cudaSuccess) e = pa_prepare<64, 2, false>();
  if (e == cudaSuccess) e = pa_prepare<64, 2, true>();
  if (e == cudaSuccess) e = pa_prepare<128, 1, true>();
  if (e == cudaSuccess) e = pa_prepare<128, 2, false>();
  if (e == cudaSuccess) e = pa_prepare<128, 2, true>();
  if (e == cudaSuccess) e = paged_attn_tc_prepare();
  return e;
}

cudaError_t launch_paged_attention(tss_paged* h, const PgAttnArgs& a, const PgBatch& batch, cudaStream_t s, bool* too_large) {
  *too_large = false;
  const int withhold = h->inject > 0;
  if (withhold) --h->inject;
  PaTask tasks[kPgMaxReq];
  for (int i = 0; i < batch.n_req; ++i) {
    const PgReq& q = batch.r[i];
    tasks[i] = PaTask{q, 0, q.first + q.n, q.first, q.n * (h->hq / h->hk), 0, 0, 0};
  }
  return pa_pass(h, a, tasks, batch.n_req, nullptr, kPaTcRows, PaWork{h->part_o, h->part_ml, h->counters, 0}, withhold, false, s, too_large);
}

// A pass over the groups' shared keys, for all rows of a group at once, then one over every request's own, which begins while
// the first one ends (it has partial results and counters of its own) and waits for it where it joins.
cudaError_t launch_paged_attention_shared(tss_paged* h, const PgAttnArgs& args, const PgBatch& batch, const PgGroups& groups, cudaStream_t s,
                                          bool* too_large) {
  *too_large = false;
  const int withhold = h->inject > 0;
  if (withhold) --h->inject;
  PgAttnArgs a = args;
  PaTask common[kPgMaxReq], mine[kPgMaxReq];
  int2 mem[kPgMaxReq];
  int n_common = 0, at = 0, n_mem = 0;
  const int gq = h->hq / h->hk;
  for (int g = 0; g < groups.n; ++g) {
    PaTask t{PgReq{0, groups.shared[g], 0, 0}, 0, groups.shared[g], 0, 0, 0, n_mem, 0};
    for (int i = at; i < at + groups.reqs[g]; ++i) {
      const PgReq& q = batch.r[i];
      mine[i] = PaTask{q, 0, q.first + q.n, q.first, q.n * gq, 0, 0, 0};
      if (q.n == 0) continue;
      if (t.members == 0) {
        t.q.seq = q.seq;
        t.q.row = q.row;
        t.from = q.first;
      }
      t.q.n += q.n;
      t.from = q.first < t.from ? q.first : t.from;
      mem[n_mem++] = make_int2(q.row, q.first);
      ++t.members;
    }
    if (t.members > 1 && groups.shared[g] > 0) {  // (alone, a request has no one to share with)
      PaReq r;
      pa_units(a, t, kPgTokens, &r);
      for (int i = at; i < at + groups.reqs[g]; ++i) {
        mine[i].k0 = groups.shared[g];
        mine[i].joins = r.units > 0;
      }
      t.rows = t.q.n * gq;
      if (r.units > 0) common[n_common++] = t;
    } else {
      n_mem -= t.members;
    }
    at += groups.reqs[g];
  }
  cudaError_t e = cudaSuccess;
  if (n_common) {
    a.own = 0;
    e = pa_pass(h, a, common, n_common, mem, kPaTcShared, PaWork{h->part_o, h->part_ml, h->counters, 0}, withhold, true, s, too_large);
  }
  if (e != cudaSuccess || *too_large) return e;
  a.own = 1;
  return pa_pass(h, a, mine, batch.n_req, mem, kPaTcShared, PaWork{h->own_o, h->own_ml, h->own_counters, n_common > 0}, withhold && !n_common, true, s,
                 too_large);
}

}  // namespace tss
