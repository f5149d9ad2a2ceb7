// Attention of wide draft blocks over the paged 4-bit cache on the 5th-generation tensor cores (tcgen05),
// head_dim 128: the operation of paged_attn.cu for more than kPaTcRows query rows of a KV head (trees, long
// chains, grouped heads), which take the MMA's 128-row side.  Per page of 64 tokens, g a group of 64 dims:
//   S_g [128 rows x 64 keys] = Q_g C_g^T            score = f (s_0 S_0 + s_1 S_1 + z_0 q_0 + z_1 q_1)
//   O_g [128 rows x 64 dims] += (P s'_g) C'_g       o = (2^9 O_g + sum_t p_t (z' + 7.5 s')_tg) / sum_t p_t
// C is K's codes as fp16 subnormals (paged_attn.cu), C' V's centred, (c - 7.5) 2^-9; scales, minima, references and sums
// are fp32, Q exact in fp16 (scaled by a power of two), the weights one fp16 part (bf16 outputs) or two.
//
// References are a row's and group's, as in paged_attn.cu; a row's two are one while they are 2 binades apart at most, so that
// pages whose groups have scales alike cost one maximum a score and no factor (61 rows over 4600 tokens 71 us, 79 with
// scales 8 or 10^6 times apart).
//
// A nibble word (8 dims of a key, or 8 keys of a dim) becomes eight values of a K-major operand by four ANDs and a
// shift; their order, and in K the factor 16 of odd nibbles, are matched in Q and P.
//
// Roles (640 threads): warp 0 copies pages (one bulk copy each), warp 1 issues MMAs, warps 2-3 expand codes
// and parameters, warps 4-19 are the softmax.  Scores lie in three buffers of TMEM, read as blocks of 16 rows and 8
// columns: a thread has 4 rows and 4 of a page's keys (in the shape of a row a thread each thread reads the parameters,
// nine floats a key, of 16 keys: four times the shared-memory traffic, 81 us where this took 75).  The weights go back
// to TMEM, over the scores that they come from, as the second product's first operand.  Operands of K and V are
// double-buffered, so a page's expansion and scores run under the softmax of the pages before it.  Runs of pages as in
// paged_attn.cu, one CTA an SM; partials of shared items are joined by the last CTA in CTA order.
// Every wait is bounded; on expiry the kernel records a timeout, drains its copies and MMAs and returns.
//
// Bound: the latency of a page's way through a softmax warp: load of the scores, 16 scores a thread, the quadrant's vote on
// its references, exponentials, store of the weights.  1.1 us a page with 32 rows in use, 1.4 us with 128; the MMAs take
// 0.3 us of it.  About 12 us more a launch: first page, masked pages, end of an item, join.  128 rows, 32 heads, four requests
// of 4600 tokens 123 us; 4 requests of 2048 .. 8000 tokens, 61 rows, 32 / 8 heads 71 us.  (At 640 threads of 96 registers some
// 64 bytes a thread spill.)  Outputs written by the threads of their rows, 8 bytes a lane, had cost 5 us an item.
// Built and slower at the latter size (when this took 75 us): 8 softmax warps of half a page each (83 us), or of every
// second page (105); a vote by a barrier that warps wait for only after their exponentials (78); K and V expanded by
// warps of their own into three buffers (85).
#include <cfloat>
#include <cstddef>
#include <type_traits>

#include "paged_attn.cuh"

namespace tss {
namespace {

constexpr int kPtD = 128, kPtRows = 128, kPtKeys = 64;
constexpr int kPtExpand = 2, kPtSoftWarps = 16;   // warps that expand codes; those of the softmax
constexpr int kPtSoft = kPtSoftWarps * 32, kPtThreads = 64 + kPtExpand * 32 + kPtSoft;
constexpr int kPtRaw = 4;                         // pages in the ring of copies
using PtBlock = PgBlock<kPtD>;
constexpr int kPtQ = kPtRows * 64 * 2;            // one group of Q: 128 rows of 128 bytes
constexpr int kPtOp = kPtKeys * 64 * 2;           // one group of C or C': 64 rows of 128 bytes
constexpr int kPtJoin = 128;                      // partials whose weights the joining of an item keeps beside Q's memory
static_assert(kPtJoin * kPtRows == kPtRows * kPtD, "the outputs of an item pass through the same memory");
constexpr int kPtParams = 9;                      // arrays of 64: s0 s1 z0 z1 of K, the same of V, log2 of V's larger scale
constexpr uint32_t kPtTmem = 512;                 // S: 3 buffers x 2 groups x 64 columns; O: 128 from column kPtO
constexpr uint32_t kPtO = 384;

struct __align__(16) PtShared {
  float par[4][kPtParams][kPtKeys];                   // keys in the order 16 q + 4 x + 2 b + e for 16 q + 8 b + 2 x + e
  uint64_t raw_full[kPtRaw], raw_free[kPtRaw], k_full[2], k_free[2], v_full[2], v_free[2], par_full[4];
  uint64_t s_full[3], p_full[3], o_done[2], q_full, o_full, drain;
  uint32_t tmem;
  int abort, last, bad[kPtRaw], bad_par[4];
  float4 row[kPtRows];                                // factor of the codes' sums, then of the minima of groups 0 and 1
  unsigned long long anc[2][kPtRows];                 // the rows of its block that a row sees
  long long out_at[kPtRows];                          // where its output begins
  int qp[kPtRows];                                    // its position
  int bp[kPgMaxRows];                                 // under a window, the positions of the block's rows
  float inv[kPtRows];                                 // 1 / sum of its weights
  float other[kPtRows];                               // what its results over shared keys are multiplied by
  float top[2][4][kPtRows];                           // maxima of its quarters, of scores and V's scales of each group
  float part[4][3][kPtRows];                          // the quarters' sums: p, p z'_0, p z'_1
};
static_assert(offsetof(PtShared, par) % 16 == 0 && offsetof(PtShared, row) % 16 == 0 && offsetof(PtShared, raw_full) % 8 == 0,
              "alignment of vectors and barriers");
constexpr size_t kPtSmem = 1024 + 2 * kPtQ + 2 * 4 * kPtOp + kPtJoin * kPtRows * 4 + kPtRaw * PtBlock::kBytes;

__host__ __device__ constexpr uint32_t idesc_f16_m128(int n) {
  return (1u << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(128 >> 4) << 24);
}

// mbar_wait, asleep between looks: sixteen warps that poll would take the issue slots of those that work.
__device__ __noinline__ bool quiet_wait_slow(uint64_t* bar, uint32_t parity, volatile int* abort, int* status) {
  const uint64_t t0 = globaltimer_ns();
  while (!mbar_try_wait_sleep(bar, parity, 20000)) {
    if (*abort) return false;
    if (globaltimer_ns() - t0 > kWaitLimitNs) {
      *abort = 1;
      report(status, kStatusTimeout);
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool quiet_wait(uint64_t* bar, uint32_t parity, volatile int* abort, int* status) {
  return mbar_try_wait(bar, parity) || quiet_wait_slow(bar, parity, abort, status);
}

// A word's eight codes as fp16 subnormals.
__device__ __forceinline__ uint4 expand(uint32_t x) {
  const uint32_t y = x >> 8;
  return make_uint4(x & 0x000f000fu, x & 0x00f000f0u, y & 0x000f000fu, y & 0x00f000f0u);
}

// 16 TMEM lanes (from taddr's) and 16 columns, left in flight (tmem_wait() before they are used): thread l has, in
// r[4 b + 2 y + e], lane l / 4 + 8 y and column 8 b + 2 (l % 4) + e.
__device__ __forceinline__ void tmem_ld_block(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
// The same layout, 8 columns, stored; tmem_stored() before another thread is told.
__device__ __forceinline__ void tmem_st_block(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.16x256b.x1.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3])
               : "memory");
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// umma_bf16 with its first operand in TMEM: 128 lanes, 8 columns of two 16-bit values.
__device__ __forceinline__ void umma_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// OR of v over the 128 threads of named barrier id.
__device__ __forceinline__ bool quad_or(int id, bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %1, 0;\n\t"
      "bar.red.or.pred p, %2, 128, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}\n"
      : "=r"(r)
      : "r"(v ? 1u : 0u), "r"(id)
      : "memory");
  return r != 0;
}

// Keys of the tile from key0 that a row sees (position qp; lo, hi: the rows of its block that it sees).
__device__ __forceinline__ unsigned long long row_sees(const PgAttnArgs& a, const PaReq& r, const int* bp, int qp, unsigned long long lo,
                                                       unsigned long long hi, int key0) {
  unsigned long long v = ~0ull, blk = 0;  // blk: bits that are rows of the block
  if (key0 + kPtKeys > r.first) {
    if (key0 < r.first) {
      const int c = r.first - key0;  // 1..63
      blk = ~0ull << c;
      v = ~blk | (lo << c);
    } else {
      const int j = key0 - r.first;  // block row of the tile's first key
      blk = ~0ull;
      v = j == 0 ? lo : j < 64 ? (lo >> j) | (hi << (64 - j)) : j < 128 ? hi >> (j - 64) : 0ull;
    }
  }
  if (a.window) {
    // (keys from qp on are near; no difference here leaves 32 bits, whatever the window)
    const int from = max(qp - key0, 0) - (a.window - 1), sinks = a.sinks - key0;
    unsigned long long near = from <= 0 ? ~0ull : from >= 64 ? 0ull : ~0ull << from;
    if (a.positions && blk) {  // a row of the block stands at its own position
      near &= ~blk;
      for (unsigned long long x = v & blk; x; x &= x - 1) {
        const int i = __ffsll(static_cast<long long>(x)) - 1;
        if (qp - bp[key0 + i - r.first] < a.window) near |= 1ull << i;
      }
    }
    v &= near | (sinks >= 64 ? ~0ull : sinks <= 0 ? 0ull : (1ull << sinks) - 1);
  }
  return v;
}

// The softmax team of an item's last CTA joins the partials of CTAs c0..c1: first every row's weights of them (in
// shared memory, some of it Q's: no MMA is in flight), then 4 dims of 8 rows a thread, their loads in flight together.
template <typename P>
__device__ __forceinline__ void join_parts(const P& p, PtShared& sh, uint8_t* sq, uint8_t* sj, const PaReq& r, int h, int row0, int rows,
                                           int c0, int c1, int sw, int qt, int row, int lane) {
  const int parts = c1 - c0 + 1;
  const auto weight = [&](int x) {
    return (x < kPtJoin ? reinterpret_cast<float*>(sj) + x * kPtRows : reinterpret_cast<float*>(sq) + (x - kPtJoin) * kPtRows);
  };
  const auto slot = [&](int x) { return static_cast<long long>((c0 + x) * 2 + (x == 0)) * kPtRows; };
  float M = -INFINITY, L = 0.f;
  if (row < rows)
#pragma unroll 4
    for (int x = qt; x < parts; x += 4) M = fmaxf(M, __ldcg(p.part_ml + slot(x) + row).x);
  sh.top[0][qt][row] = M;
  named_bar_sync(5, kPtSoft);
  M = fmaxf(fmaxf(sh.top[0][0][row], sh.top[0][1][row]), fmaxf(sh.top[0][2][row], sh.top[0][3][row]));
  const float mb = M == -INFINITY ? 0.f : M;
  if (row < rows)
#pragma unroll 4
    for (int x = qt; x < parts; x += 4) {
      const float2 ml = __ldcg(p.part_ml + slot(x) + row);
      const float w = ex2(ml.x - mb);
      L = fmaf(w, ml.y, L);
      weight(x)[row] = w;
    }
  sh.part[qt][0][row] = L;
  named_bar_sync(5, kPtSoft);
  constexpr int kRowsOf = kPtRows / kPtSoftWarps;
  float4 o[kRowsOf];
#pragma unroll
  for (int i = 0; i < kRowsOf; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
  for (int x = 0; x < parts; ++x) {
    float4 y[kRowsOf];
#pragma unroll
    for (int i = 0; i < kRowsOf; ++i) {
      const int q = sw + i * kPtSoftWarps;
      y[i] = q < rows ? __ldcg(reinterpret_cast<const float4*>(p.part_o + (slot(x) + q) * kPtD) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int i = 0; i < kRowsOf; ++i) {
      const int q = sw + i * kPtSoftWarps;
      if (q >= rows) continue;
      const float w = weight(x)[q];
      o[i].x = fmaf(w, y[i].x, o[i].x);
      o[i].y = fmaf(w, y[i].y, o[i].y);
      o[i].z = fmaf(w, y[i].z, o[i].z);
      o[i].w = fmaf(w, y[i].w, o[i].w);
    }
  }
  wait_for_shared(p);
#pragma unroll
  for (int i = 0; i < kRowsOf; ++i) {
    const int q = sw + i * kPtSoftWarps;
    if (q >= rows) continue;
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m = fmaxf(m, sh.top[0][k][q]);
      l += sh.part[k][0][q];
    }
    finish_row<kPtD>(p, r, h, row0 + q, lane, m, l, o[i]);
  }
}

// TWO: weights of two fp16 parts (fp16 outputs); else one (bf16 outputs: its 2^-12 is a fraction of their own 2^-9).  SH: a pass
// of the attention of sequences that share keys.
template <bool TWO, bool SH>
__global__ void __launch_bounds__(kPtThreads, 1) paged_attn_tc_kernel(const __grid_constant__ typename PaParamsOf<SH>::type p) {
  extern __shared__ uint8_t pt_dyn[];
  __shared__ PtShared sh;
  const uint32_t skew = (1024 - (smem_u32(pt_dyn) & 1023)) & 1023;
  uint8_t* sq = pt_dyn + skew;        // Q: group 0, group 1
  uint8_t* skv = sq + 2 * kPtQ;       // [buffer] C_0, C_1, C'_0, C'_1
  uint8_t* sj = skv + 2 * 4 * kPtOp;  // weights of partials; outputs on their way
  uint8_t* raw = sj + kPtJoin * kPtRows * 4;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const PgAttnArgs& a = p.a;
  const int gq = a.hq / a.hk;
  int u0, u1, first_cta, splits;
  cta_run(p, &u0, &u1, &first_cta, &splits);
  if (tid == 0) {
    for (int i = 0; i < kPtRaw; ++i) {
      mbar_init(&sh.raw_full[i], 1);
      mbar_init(&sh.raw_free[i], kPtExpand);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.k_full[i], kPtExpand);
      mbar_init(&sh.k_free[i], 1);
      mbar_init(&sh.v_full[i], kPtExpand);
      mbar_init(&sh.v_free[i], 1);
      mbar_init(&sh.o_done[i], 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(&sh.par_full[i], kPtExpand);
    for (int i = 0; i < 3; ++i) {
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.p_full[i], kPtSoftWarps);
    }
    mbar_init(&sh.q_full, kPtSoftWarps);
    mbar_init(&sh.o_full, 1);
    mbar_init(&sh.drain, 1);
    sh.abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&sh.tmem, kPtTmem);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // Each role waits for the kernel before this one: before it meets global memory, and before waits that are bounded.
  const auto ready = [&] {
    if constexpr (SH) {
      if (!p.early) griddep_wait();  // (what it reads before that was complete when the pass before it began)
    } else {
      griddep_wait();
    }
    griddep_launch();
  };
  const uint32_t tm = sh.tmem;
  volatile int* abort = &sh.abort;
  const int n = u1 - u0;  // pages of the run; page t of it is unit u0 + t
  const auto request_of = [&](int u) {
    int b = 0;
    while (b + 1 < p.n_req && p.r[b + 1].off <= u) ++b;
    return b;
  };

  if (warp == 0) {
    // ---------------- pages: the table's entries 32 at a time, one bulk copy a page ----------------
    int t = 0;
    bool ok = true;
    for (int t0 = 0; t0 < n && ok; t0 += 32) {
      long long blk = -1, place = -1;
      int h = 0;
      if (t0 + lane < n) {
        const int u = u0 + t0 + lane;
        const PaReq& r = p.r[request_of(u)];
        const int v = u - r.off, item = v / r.units, x = v - item * r.units, at = x < r.sink ? x : x - r.sink + r.lo;
        place = static_cast<long long>(r.seq) * a.max_pages + at;
        h = item % a.hk;
      }
      if (t0 == 0) ready();
      if (place >= 0) {
        const int page = __ldcg(a.table + place);
        if (page >= 0 && page < a.n_pages)
          blk = static_cast<long long>(page) * a.hk + h;
        else
          report(a.status, kStatusCheck);
      }
      for (int k = 0; k < 32 && t < n; ++k, ++t) {
        const long long src = __shfl_sync(0xffffffffu, blk, k);
        const int s = t % kPtRaw;
        ok = __all_sync(0xffffffffu, t < kPtRaw || quiet_wait(&sh.raw_free[s], ((t / kPtRaw) - 1) & 1, abort, a.status));
        if (!ok) break;
        if (lane == 0) {
          sh.bad[s] = src < 0;
          if (src < 0) {
            mbar_arrive(&sh.raw_full[s]);
          } else {
            mbar_arrive_expect_tx(&sh.raw_full[s], PtBlock::kBytes);
            bulk_load(raw + s * PtBlock::kBytes, a.pool + src * PtBlock::kBytes, PtBlock::kBytes, &sh.raw_full[s]);
          }
        }
      }
    }
    // the copies issued last have landed before the kernel returns
    for (int k = max(0, t - kPtRaw); k < t; ++k) mbar_drain(&sh.raw_full[k % kPtRaw], (k / kPtRaw) & 1);
  } else if (warp == 1) {
    // ---------------- MMAs: S two pages ahead, then O += P C' ----------------
    ready();
    // (issued behind elect.sync: 4 trees of 33 rows over a shared prefix 117 -> 108 us; not so in the kernel of single requests, where
    // 4 trees of 61 rows took 74 us instead of 72)
    if (SH ? elect_one() : lane == 0) {
      constexpr uint32_t id = idesc_f16_m128(64);
      const uint32_t q_a = smem_u32(sq), kv_a = smem_u32(skv);
      bool ok = true;
      for (int t = 0, seg = 0; t < n && ok; ++seg) {
        const PaReq& r = p.r[request_of(u0 + t)];
        const int len = min(n - t, r.units - (u0 + t - r.off) % r.units);
        const auto scores = [&](int u) {
          const int s = u & 1, b = u % 3;
          // (buffer b's last reader, P V of page u - 3, was issued before: MMAs run in the order of their issue)
          if (!mbar_wait(&sh.k_full[s], (u >> 1) & 1, abort, a.status)) return false;
          tc_fence_after();
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              umma_bf16(tm + b * 128 + g * 64, sdesc_sw128(q_a + g * kPtQ + k * 32), sdesc_sw128(kv_a + (s * 4 + g) * kPtOp + k * 32), id,
                        k ? 1u : 0u);
          umma_commit(&sh.s_full[b]);
          umma_commit(&sh.k_free[s]);
          return true;
        };
        if (p.withhold && blockIdx.x == 0) break;
        ok = mbar_wait(&sh.q_full, seg & 1, abort, a.status) && scores(t) && (len < 2 || scores(t + 1));
        for (int j = 0; ok && j < len; ++j) {
          const int u = t + j, s = u & 1, b = u % 3;
          ok = mbar_wait(&sh.v_full[s], (u >> 1) & 1, abort, a.status) && mbar_wait(&sh.p_full[b], (u / 3) & 1, abort, a.status);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int part = 0; part < (TWO ? 2 : 1); ++part)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                umma_ta(tm + kPtO + g * 64, tm + b * 128 + g * 64 + k * 16 + part * 8, sdesc_sw128(kv_a + (s * 4 + 2 + g) * kPtOp + k * 32), id,
                        (j || part || k) ? 1u : 0u);
          umma_commit(&sh.o_done[u & 1]);
          umma_commit(&sh.v_free[s]);
          if (j == len - 1) umma_commit(&sh.o_full);
          ok = j + 2 >= len || scores(u + 2);
        }
        t += len;
      }
      // every MMA issued has completed before the kernel returns
      umma_commit(&sh.drain);
      mbar_drain(&sh.drain, 0);
    }
  } else if (warp < 2 + kPtExpand) {
    // ---------------- codes to operands, parameters to fp32 ----------------
    // A lane's units of a page are 16 keys (dims) apart, so that its chunks' places differ by constants.
    ready();
    const int x = tid - 64;
    constexpr int kTurns = 256 / (32 * kPtExpand);
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (int t = 0; t < n; ++t) {
      const int s = t & 1, rs = t % kPtRaw;
      const uint8_t* blk = raw + rs * PtBlock::kBytes;
      uint8_t* op = skv + s * 4 * kPtOp;
      if (!__all_sync(0xffffffffu, quiet_wait(&sh.raw_full[rs], (t / kPtRaw) & 1, abort, a.status) &&
                                       (t < 2 || quiet_wait(&sh.k_free[s], ((t >> 1) - 1) & 1, abort, a.status))))
        break;
      const bool bad = sh.bad[rs];  // without a page: zeros, so that no weight meets a stale operand
      // Parameters, in a buffer of four: page t - 4's are read out, since S(t - 2), which is complete, was issued after
      // P V of page t - 4.
      if (x < kPtKeys) {
        const uint2 kp = *reinterpret_cast<const uint2*>(blk + PtBlock::kKParams + 8 * x);
        const uint2 vp = *reinterpret_cast<const uint2*>(blk + PtBlock::kVParams + 8 * x);
        const auto pair = [](uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); };
        const float2 k0 = pair(kp.x), k1 = pair(kp.y), v0 = pair(vp.x), v1 = pair(vp.y);
        const int at = (x & 48) | (x & 6) << 1 | (x & 8) >> 2 | (x & 1);
        const float all[kPtParams] = {k0.x, k1.x, k0.y, k1.y, v0.x, v1.x, fmaf(v0.x, 7.5f, v0.y), fmaf(v1.x, 7.5f, v1.y), __log2f(fmaxf(fmaxf(v0.x, v1.x), kLeast))};
#pragma unroll
        for (int i = 0; i < kPtParams; ++i) sh.par[t & 3][i][at] = all[i];
        if (x == 0) sh.bad_par[t & 3] = bad;
      }
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        // unit w: key w / 4, dims 16 (w % 4) .. + 15 of each group
        const int w = i * 32 * kPtExpand + x, key = w >> 2, c = 2 * (w & 3);
        const uint4 k = bad ? zero : *reinterpret_cast<const uint4*>(blk + PtBlock::kK + w * 16);
        uint8_t *k0 = op + key * 128 + ((c ^ (key & 7)) << 4), *k1 = op + key * 128 + (((c + 1) ^ (key & 7)) << 4);
        *reinterpret_cast<uint4*>(k0) = expand(k.x);
        *reinterpret_cast<uint4*>(k1) = expand(k.y);
        *reinterpret_cast<uint4*>(k0 + kPtOp) = expand(k.z);
        *reinterpret_cast<uint4*>(k1 + kPtOp) = expand(k.w);
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&sh.par_full[t & 3]);
        mbar_arrive(&sh.k_full[s]);
      }
      if (!__all_sync(0xffffffffu, t < 2 || quiet_wait(&sh.v_free[s], ((t >> 1) - 1) & 1, abort, a.status))) break;
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        // unit w: half w / 128, dims 4 (w / 4 % 32) .. + 3, tokens 8 b + 2 (w % 4) + i of the half; b = 0, 1 go to the
        // half's first quarter (16 keys: two chunks of a dim's row), b = 2, 3 to its second, as 8 bytes at w % 4.  (Lanes
        // of every second pair of dims' groups take the quarters in the other order, to meet other banks.)
        const int w = i * 32 * kPtExpand + x, d0 = ((w >> 2) & 31) * 4, swap = (w >> 3) & 1;
        const uint4 v = bad ? zero : *reinterpret_cast<const uint4*>(blk + PtBlock::kV + w * 16);
        uint8_t* vd = op + (2 + d0 / 64) * kPtOp + (d0 % 64) * 128 + (w & 1) * 8;
        const int vc = (w >> 7) * 4 + ((w & 3) >> 1), first = vc + 2 * swap, second = vc + 2 - 2 * swap;
        const uint32_t vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t f = vw[e] >> (8 * swap), g = vw[e] >> (8 - 8 * swap);
          uint8_t* row = vd + e * 128;
          *reinterpret_cast<uint2*>(row + ((first ^ ((d0 + e) & 7)) << 4)) = make_uint2(centre(f & 0x000f000fu, false), centre(f & 0x00f000f0u, true));
          *reinterpret_cast<uint2*>(row + ((second ^ ((d0 + e) & 7)) << 4)) = make_uint2(centre(g & 0x000f000fu, false), centre(g & 0x00f000f0u, true));
        }
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&sh.v_full[s]);
        mbar_arrive(&sh.raw_free[rs]);
      }
    }
  } else {
    // ---------------- softmax: warp = (32 rows, a quarter of a page's keys) ----------------
    // Thread: rows qd * 32 + r4 + 8 i, keys 16 qt + 8 b + 2 x4 + e of a page, so that it reads a quarter of the keys'
    // parameters.  Its weights go where its quarter's scores were, as the second product's operand in TMEM: words b of
    // x4 at columns 2 x4 + b.  Queries and outputs: row qd * 32 + lane.
    // After a wait that gave up the threads go on without waiting, through the same barriers.
    const int sw = warp - 2 - kPtExpand, qd = warp & 3, qt = sw >> 2, half = qt >> 1;
    const int row = qd * 32 + lane, quad = 1 + qd, r4 = lane >> 2, x4 = lane & 3;
    const uint32_t lanes = static_cast<uint32_t>(qd * 32) << 16;
    const auto of_row = [&](const float* v) {  // row `lane`'s value, from a thread that has it
      float y = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float z = __shfl_sync(0xffffffffu, v[i], 4 * (lane & 7));
        if (i == lane >> 3) y = z;
      }
      return y;
    };
    bool ok = true;
    for (int t = 0, seg = 0; t < n; ++seg) {
      const int rb = request_of(u0 + t);
      const PaReq& r = p.r[rb];
      const int v = u0 + t - r.off, item = v / r.units, x0 = v - item * r.units, len = min(n - t, r.units - x0);
      const int h = item % a.hk, row0 = item / a.hk * kPtRows, rows = min(kPtRows, r.n * gq - row0);
      if (seg == 0) ready();
      // Q: 16 lanes a row, 8 dims each, as chunks in the operand's order; the warp's rows in flight together
      constexpr int kTurns = kPtRows / 2 / kPtSoftWarps;
      uint4 rawq[kTurns];
      const int c8 = lane & 15;
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int qr = (sw * kTurns + i) * 2 + (lane >> 4), q = row0 + qr;
        rawq[i] = make_uint4(0, 0, 0, 0);
        if (qr < rows)
          rawq[i] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + (r.row + q / gq) * a.qs +
                                                    static_cast<long long>(h * gq + q % gq) * kPtD + c8 * 8);
      }
#pragma unroll
      for (int i = 0; i < kTurns; ++i) {
        const int qr = (sw * kTurns + i) * 2 + (lane >> 4);
        const uint32_t in[4] = {rawq[i].x, rawq[i].y, rawq[i].z, rawq[i].w};
        float x[8], big = 0.f, sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = a.is_half ? __half22float2(*reinterpret_cast<const __half2*>(&in[e]))
                                     : make_float2(__uint_as_float(in[e] << 16), __uint_as_float(in[e] & 0xffff0000u));
          x[2 * e] = f.x;
          x[2 * e + 1] = f.y;
          big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
          sum += f.x + f.y;
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float up = query_scale(big);
        const float lo = up * 0.0625f;
        const uint4 w = make_uint4(pack_f16(x[0] * up, x[4] * up), pack_f16(x[1] * lo, x[5] * lo), pack_f16(x[2] * up, x[6] * up),
                                   pack_f16(x[3] * lo, x[7] * lo));
        *reinterpret_cast<uint4*>(sq + (c8 >> 3) * kPtQ + qr * 128 + (((c8 & 7) ^ (qr & 7)) << 4)) = w;
        const float z1 = __shfl_down_sync(0xffffffffu, sum, 8);
        if (c8 == 0) sh.row[qr] = make_float4(a.scale_log2 * 16777216.f / up, sum * a.scale_log2, z1 * a.scale_log2, 0.f);
      }
      const bool valid = row < rows, active = qd * 32 < rows;
      int qp = 0;
      unsigned long long anc_lo = ~0ull, anc_hi = ~0ull;
      if (valid) {
        const int ti = (row0 + row) / gq;
        qp = row_position(p, r, ti);
        if (SH && !a.own) {  // (no shared key is of a row's block)
        } else if (a.mask) {
          anc_lo = __ldcg(a.mask + 2LL * (r.row + ti));
          anc_hi = __ldcg(a.mask + 2LL * (r.row + ti) + 1);
        } else {
          anc_lo = ti >= 63 ? ~0ull : (2ull << ti) - 1;
          anc_hi = ti < 64 ? 0ull : ti == 127 ? ~0ull : (2ull << (ti - 64)) - 1;
        }
        // (rows that the block does not have are not seen, whatever the mask says; a group's rows may be more than 128)
        if (r.n < 64) anc_lo &= (1ull << r.n) - 1;
        anc_hi = r.n <= 64 ? 0ull : r.n < 128 ? anc_hi & ((1ull << (r.n - 64)) - 1) : anc_hi;
      }
      // (four trees of 33 rows in a window over a shared prefix: 144 us where every masked page's rows read them from memory, 118 so)
      if (a.positions && sw * 32 + lane < min(r.n, kPgMaxRows))
        sh.bp[sw * 32 + lane] = max(__ldcg(a.positions + r.row + sw * 32 + lane), r.first);
      if (qt == 0) {
        sh.qp[row] = qp;
        sh.anc[0][row] = anc_lo;
        sh.anc[1][row] = anc_hi;
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.q_full);
      named_bar_sync(5, kPtSoft);
      int pmax = 0;
      if (a.window) {
        pmax = valid ? qp : 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) pmax = max(pmax, __shfl_xor_sync(0xffffffffu, pmax, o));
      }
      int all0, all1, all2;
      units_in_sight(a, r, kPtKeys, pmax, &all0, &all1, &all2);
      float ref[4];  // of the first group of dims, and the factor from weights under it to those under the second's
      float fx[4];
      bool split = false;  // some row's factor is not 1
      f2_t l2[4], oz0[4], oz1[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ref[i] = -FLT_MAX;  // (nothing seen)
        fx[i] = 1.f;
        l2[i] = oz0[i] = oz1[i] = f2_pack(0.f, 0.f);
      }
      for (int j = 0; j < len; ++j) {
        const int u = t + j, sb = u % 3;
        ok = ok && quiet_wait(&sh.par_full[u & 3], (u >> 2) & 1, abort, a.status) && quiet_wait(&sh.s_full[sb], (u / 3) & 1, abort, a.status);
        tc_fence_after();
        if (active) {
          const int x = x0 + j;
          uint32_t vis = 0xffffu;  // bit 4 i + 2 b + e
          if (sh.bad_par[u & 3]) {
            vis = 0u;
          } else if (!(x < all0 || (x >= all1 && x < all2))) {
            const int key0 = (x < r.sink ? x : x - r.sink + r.lo) * kPtKeys;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int q = qd * 32 + r4 + 8 * i;
              if (q >= rows) continue;
              const uint32_t m = static_cast<uint32_t>(row_sees(a, r, sh.bp, sh.qp[q], sh.anc[0][q], sh.anc[1][q], key0) >> (16 * qt)) >> (2 * x4);
              vis &= ~(15u << (4 * i)) | (m & 3u) << (4 * i) | (m >> 8 & 3u) << (4 * i + 2);
            }
          }
          const auto page = [&](auto all_tag) {
            constexpr bool kAll = decltype(all_tag)::value;  // the thread's rows see all of its keys
            const float* par = &sh.par[u & 3][0][16 * qt + 4 * x4];
            const auto pr = [&](int k) {  // .x: block 0's keys, .y: block 1's
              return *reinterpret_cast<const ulonglong2*>(par + k * kPtKeys);
            };
            const uint32_t at = tm + lanes + sb * 128 + 16 * qt;
            f2_t c[4][2];  // scores
            {
              const ulonglong2 a0 = pr(0), a1 = pr(1), b0 = pr(2), b1 = pr(3);
              __syncwarp();
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                uint32_t s0[8], s1[8];
                tmem_ld_block(at + (static_cast<uint32_t>(16 * h) << 16), s0);
                tmem_ld_block(at + (static_cast<uint32_t>(16 * h) << 16) + 64, s1);
                tmem_wait();
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                  const float4 q = sh.row[qd * 32 + r4 + 8 * (2 * h + y)];
                  const f2_t f2 = f2_pack(q.x, q.x), zq0 = f2_pack(q.y, q.y), zq1 = f2_pack(q.z, q.z);
#pragma unroll
                  for (int b = 0; b < 2; ++b) {
                    const uint32_t *m = &s0[4 * b + 2 * y], *z = &s1[4 * b + 2 * y];
                    const f2_t m2 = f2_pack(__uint_as_float(m[0]), __uint_as_float(m[1])), z2 = f2_pack(__uint_as_float(z[0]), __uint_as_float(z[1]));
                    const f2_t code = f2_fma(b ? a1.y : a1.x, z2, f2_mul(b ? a0.y : a0.x, m2));
                    c[2 * h + y][b] = f2_fma(code, f2, f2_fma(b ? b1.y : b1.x, zq1, f2_mul(b ? b0.y : b0.x, zq0)));
                  }
                }
              }
            }
            // maxima over the thread's keys of a row's scores, each more lg(block).x or .y
            const auto tops = [&](float* top, auto lg) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                top[i] = -INFINITY;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                  const float2 e = f2_unpack(f2_add(c[i][b], lg(b)));
                  if constexpr (kAll) {
                    top[i] = fmaxf(top[i], fmaxf(e.x, e.y));
                  } else {
                    top[i] = fmaxf(top[i], vis >> (4 * i + 2 * b) & 1u ? e.x : -INFINITY);
                    top[i] = fmaxf(top[i], vis >> (4 * i + 2 * b + 1) & 1u ? e.y : -INFINITY);
                  }
                }
              }
            };
            const auto tops_of = [&](float* top, int g) {  // with V's scales of group g
              const ulonglong2 s = pr(4 + g);
              const auto log2_of = [](f2_t x) {
                const float2 q = f2_unpack(x);
                return f2_pack(__log2f(fmaxf(q.x, kLeast)), __log2f(fmaxf(q.y, kLeast)));
              };
              const f2_t lo = log2_of(s.x), hi = log2_of(s.y);
              tops(top, [&](int b) { return b ? hi : lo; });
            };
            const auto second = [&](int i) { return ref[i] - static_cast<float>((__float_as_int(fx[i]) >> 23) - 127); };  // its reference
            bool over = false;
            if (split) {
              float top[4];
              tops_of(top, 0);
#pragma unroll
              for (int i = 0; i < 4; ++i) over |= top[i] - ref[i] > 15.f;
              tops_of(top, 1);
#pragma unroll
              for (int i = 0; i < 4; ++i) over |= top[i] - second(i) > 15.f;
            } else {
              float top[4];
              const ulonglong2 lg = pr(8);
              tops(top, [&](int b) { return b ? lg.y : lg.x; });
#pragma unroll
              for (int i = 0; i < 4; ++i) over |= top[i] - ref[i] > 15.f;
            }
            // A row's references rise where a weight times its value's scale would pass 2^15, to leave each group's largest
            // between 2^6 and 2^7 (whole numbers, so that the factor between the groups is a power of two; one for both, and a
            // largest of up to 2^9, where they are 2 apart at most).
            if (quad_or(quad, over)) {
              float top[2][4];
#pragma unroll
              for (int g = 0; g < 2; ++g) {
                tops_of(top[g], g);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  top[g][i] = fmaxf(top[g][i], __shfl_xor_sync(0xffffffffu, top[g][i], 1));
                  top[g][i] = fmaxf(top[g][i], __shfl_xor_sync(0xffffffffu, top[g][i], 2));
                  if (x4 == 0) sh.top[g][qt][qd * 32 + r4 + 8 * i] = top[g][i];
                }
              }
              named_bar_sync(quad, 128);
              bool moved = false;
              float al[4];  // of the group of dims that the thread's outputs are of
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int q = qd * 32 + r4 + 8 * i;
                al[i] = 1.f;
                float was[2] = {ref[i], second(i)}, now[2];
                bool up = false;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                  const float most = fmaxf(fmaxf(sh.top[g][0][q], sh.top[g][1][q]), fmaxf(sh.top[g][2][q], sh.top[g][3][q]));
                  up |= most - was[g] > 15.f;
                  now[g] = fmaxf(was[g], ceilf(most - 7.f));
                }
                if (up) {
                  if (fabsf(now[0] - now[1]) <= 2.f) now[0] = now[1] = fminf(now[0], now[1]);
                  const float down = pow2(was[0] - now[0]);
                  const f2_t d2 = f2_pack(down, down);
                  l2[i] = f2_mul(l2[i], d2);
                  oz0[i] = f2_mul(oz0[i], d2);
                  oz1[i] = f2_mul(oz1[i], d2);
                  ref[i] = now[0];
                  fx[i] = pow2(now[0] - now[1]);
                  al[i] = half ? pow2(was[1] - now[1]) : down;
                }
                moved |= al[i] != 1.f;
              }
              split = __any_sync(0xffffffffu, fx[0] != 1.f || fx[1] != 1.f || fx[2] != 1.f || fx[3] != 1.f);
              if (j > 0 && __any_sync(0xffffffffu, moved)) {
                ok = ok && quiet_wait(&sh.o_done[(u - 1) & 1], ((u - 1) >> 1) & 1, abort, a.status);
                const float mine = of_row(al);
                tc_fence_after();
                __syncwarp();
                float o[16];
#pragma unroll
                for (int x2 = 0; x2 < 2; ++x2) {
                  const uint32_t to = tm + lanes + kPtO + qt * 32 + x2 * 16;
                  tmem_ld16(to, o);
#pragma unroll
                  for (int i = 0; i < 16; ++i) o[i] *= mine;
                  tmem_st16(to, o);
                }
              }
            }
            const auto weigh = [&](auto split_tag) {
              constexpr bool kSplit = decltype(split_tag)::value;
              const ulonglong2 v0s = pr(4), v1s = pr(5), z0s = pr(6), z1s = pr(7);
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                uint32_t hi[2][4], lo[2][4];  // [group][2 y + b]: row i = 2 h + y
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                  const int i = 2 * h + y;
                  const f2_t nref = f2_pack(-ref[i], -ref[i]);
                  const f2_t fx2 = f2_pack(fx[i], fx[i]);
#pragma unroll
                  for (int b = 0; b < 2; ++b) {
                    const float2 e = f2_unpack(f2_add(c[i][b], nref));
                    const float2 wf = make_float2(ex2(e.x), ex2(e.y));
                    const f2_t v0 = b ? v0s.y : v0s.x, v1 = b ? v1s.y : v1s.x, z0 = b ? z0s.y : z0s.x, z1 = b ? z1s.y : z1s.x;
                    f2_t p0, p1;
                    if constexpr (kAll) {
                      f2_t w = f2_pack(wf.x, wf.y);
                      l2[i] = f2_add(l2[i], w);
                      oz0[i] = f2_fma(w, z0, oz0[i]);
                      oz1[i] = f2_fma(w, z1, oz1[i]);
                      p0 = f2_mul(w, v0);
                      p1 = f2_mul(kSplit ? f2_mul(w, fx2) : w, v1);
                    } else {  // (what a row does not see may be NaN: selected away, not multiplied)
                      const bool on0 = vis >> (4 * i + 2 * b) & 1u, on1 = vis >> (4 * i + 2 * b + 1) & 1u;
                      const auto pick = [&](f2_t m) {
                        const float2 q = f2_unpack(m);
                        return f2_pack(on0 ? q.x : 0.f, on1 ? q.y : 0.f);
                      };
                      f2_t w = f2_pack(on0 ? wf.x : 0.f, on1 ? wf.y : 0.f);
                      l2[i] = f2_add(l2[i], w);
                      oz0[i] = f2_fma(w, pick(z0), oz0[i]);
                      oz1[i] = f2_fma(w, pick(z1), oz1[i]);
                      p0 = f2_mul(w, pick(v0));
                      p1 = f2_mul(kSplit ? f2_mul(w, fx2) : w, pick(v1));
                    }
                    const auto split = [&](f2_t m, uint32_t* first, uint32_t* rest) {
                      const float2 q = f2_unpack(m);
                      *first = pack_f16(q.x, q.y);
                      if constexpr (TWO) {
                        const float2 back = __half22float2(*reinterpret_cast<const __half2*>(first));
                        const float2 d = f2_unpack(f2_fma(f2_pack(back.x, back.y), f2_pack(-1.f, -1.f), m));
                        *rest = pack_f16(d.x, d.y);
                      }
                    };
                    split(p0, &hi[0][2 * y + b], &lo[0][2 * y + b]);
                    split(p1, &hi[1][2 * y + b], &lo[1][2 * y + b]);
                  }
                }
                const uint32_t to = at + (static_cast<uint32_t>(16 * h) << 16);
                __syncwarp();
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                  tmem_st_block(to + g * 64, hi[g]);
                  if constexpr (TWO) tmem_st_block(to + g * 64 + 8, lo[g]);
                }
              }
            };
            if (split)
              weigh(std::true_type{});
            else
              weigh(std::false_type{});
            tmem_stored();
          };
          if (__all_sync(0xffffffffu, vis == 0xffffu))
            page(std::true_type{});
          else
            page(std::false_type{});
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full[sb]);  // (of a quadrant without rows: the arrival alone)
      }
      // ---- the segment's end: 32 dims a thread ----
      ok = ok && quiet_wait(&sh.o_full, seg & 1, abort, a.status);
      __syncwarp();
      tc_fence_after();
      const bool whole = x0 == 0 && len == r.units;
      if (whole) wait_for_shared(p);  // (else the join does)
      int c0 = first_cta, c1 = first_cta + splits - 1;
      if (!whole && !p.aligned) {
        c0 = cta_of_unit(p, rb, u0 + t - x0);
        c1 = cta_of_unit(p, rb, u0 + t - x0 + r.units - 1);
      }
      if (active) {
        const auto both = [](f2_t x) {
          const float2 q = f2_unpack(x);
          return q.x + q.y;
        };
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float sums[3] = {both(l2[i]), both(oz0[i]), both(oz1[i])};
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            sums[k] += __shfl_xor_sync(0xffffffffu, sums[k], 1);
            sums[k] += __shfl_xor_sync(0xffffffffu, sums[k], 2);
            if (x4 == 0) sh.part[qt][k][qd * 32 + r4 + 8 * i] = sums[k];
          }
        }
        const float my_ref = of_row(ref), my_fx = of_row(fx);
        const float m = half ? __uint_as_float(((9u + 254u) << 23) - __float_as_uint(my_fx)) : 512.f;  // 2^9 over the group's factor
        named_bar_sync(quad, 128);
        float L = 0.f, z = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          L += sh.part[i][0][row];
          z += sh.part[i][1 + half][row];
        }
        const long long slot = (blockIdx.x * 2 + (x0 == 0 ? 1 : 0)) * static_cast<long long>(kPtRows);
        if (qt == 0 && valid) {
          const int q = row0 + row, head = h * gq + q % gq;
          const long long tok = r.row + q / gq;
          sh.out_at[row] = tok * a.os + static_cast<long long>(head) * kPtD;
          if constexpr (SH) {
            float M = my_ref, sum = L, w = 1.f, v = 0.f;
            if (whole && !a.own) {
              __stcg(a.share_ml + tok * a.hq + head, make_float2(my_ref, L));
              sh.out_at[row] = (tok * a.hq + head) * kPtD;
            } else if (whole && p.joins[rb]) {
              const float2 ml = __ldcg(a.share_ml + tok * a.hq + head);
              M = fmaxf(my_ref, ml.x);
              w = ex2(my_ref - M);
              v = ex2(ml.x - M);
              sum = fmaf(v, ml.y, w * L);
            }
            const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
            sh.inv[row] = w * inv;
            sh.other[row] = v * inv;
            if (!whole)
              __stcg(p.part_ml + slot + row, make_float2(my_ref, L));
            else if (a.own && a.lse)
              a.lse[tok * a.hq + head] = (M + log2f(sum)) * 0.6931471805599453f;
          } else {
            sh.inv[row] = L > 0.f ? 1.f / L : L == 0.f ? 0.f : L;  // (a NaN stays one)
            if (!whole)
              __stcg(p.part_ml + slot + row, make_float2(my_ref, L));
            else if (a.lse)
              a.lse[tok * a.hq + head] = (my_ref + log2f(L)) * 0.6931471805599453f;
          }
        }
        // through shared memory (16-byte chunks permuted by row), so that a warp's store is a row
        float4* rows_of = reinterpret_cast<float4*>(sj) + qd * 32 * (kPtD / 4);
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
          float o[16];
          __syncwarp();
          tmem_ld16(tm + lanes + kPtO + qt * 32 + c * 16, o);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            rows_of[lane * (kPtD / 4) + ((qt * 8 + c * 4 + i) ^ lane)] =
                make_float4(fmaf(o[4 * i], m, z), fmaf(o[4 * i + 1], m, z), fmaf(o[4 * i + 2], m, z), fmaf(o[4 * i + 3], m, z));
        }
        tc_fence_before();
        named_bar_sync(quad, 128);
#pragma unroll 4
        for (int i = 0; i < 8; ++i) {
          const int ql = qt * 8 + i, q = qd * 32 + ql;
          if (q >= rows) break;
          const float4 x = rows_of[ql * (kPtD / 4) + (lane ^ ql)];
          if (SH && whole && !a.own) {
            __stcg(reinterpret_cast<float4*>(a.share_o + sh.out_at[q]) + lane, x);
          } else if (whole) {
            const float inv = sh.inv[q];
            float y[4] = {x.x * inv, x.y * inv, x.z * inv, x.w * inv};
            const long long to = sh.out_at[q] + 4 * lane;
            if constexpr (SH) {
              if (p.joins[rb]) {
                const int q2 = row0 + q;
                const long long at = (static_cast<long long>(r.row + q2 / gq) * a.hq + h * gq + q2 % gq) * kPtD;
                const float4 z = __ldcg(reinterpret_cast<const float4*>(a.share_o + at) + lane);
                const float v = sh.other[q];
                y[0] = fmaf(v, z.x, y[0]);
                y[1] = fmaf(v, z.y, y[1]);
                y[2] = fmaf(v, z.z, y[2]);
                y[3] = fmaf(v, z.w, y[3]);
              }
            }
            if (a.is_half)
              store_vec<__half, 4>(static_cast<__half*>(a.out) + to, y);
            else
              store_vec<__nv_bfloat16, 4>(static_cast<__nv_bfloat16*>(a.out) + to, y);
          } else {
            __stcg(reinterpret_cast<float4*>(p.part_o + (slot + q) * kPtD) + lane, x);
          }
        }
      }
      named_bar_sync(5, kPtSoft);
      if (!whole) {
        if (sw == 0 && lane == 0) {
          sh.last = atom_add_acq_rel_gpu(&p.counters[c0], 1) == c1 - c0;
          if (sh.last) atomicExch(&p.counters[c0], 0);
        }
        named_bar_sync(5, kPtSoft);
        if (sh.last) join_parts(p, sh, sq, sj, r, h, row0, rows, c0, c1, sw, qt, row, lane);
        named_bar_sync(5, kPtSoft);
      }
      t += len;
    }
  }
  __syncwarp();  // (lanes that wait for the other kernel would keep the one that issues MMAs from running)
  wait_for_shared(p);  // (the kernel ends no earlier than the one before it)
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tm, kPtTmem);
  }
}

}  // namespace

template <bool TWO>
cudaError_t pt_prepare() {
  const int bytes = static_cast<int>(kPtSmem);
  const cudaError_t e = cudaFuncSetAttribute(paged_attn_tc_kernel<TWO, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  return e == cudaSuccess ? cudaFuncSetAttribute(paged_attn_tc_kernel<TWO, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) : e;
}
cudaError_t paged_attn_tc_prepare() {
  const cudaError_t e = pt_prepare<false>();
  return e == cudaSuccess ? pt_prepare<true>() : e;
}

cudaError_t launch_paged_attention_tc(PaShared& p, bool shared, int sms, cudaStream_t s) {
  // (two pages at least, so that the copy, the expansion and the scores of one run under the other's softmax; an
  // item's start and end cost about as much as 6)
  const int grid = pa_cut(p, sms, 2, 6, 6);
  const dim3 g(grid), b(kPtThreads);
  if (shared) return launch_k(p.a.is_half ? paged_attn_tc_kernel<true, true> : paged_attn_tc_kernel<false, true>, g, b, kPtSmem, s, true, p);
  return launch_k(p.a.is_half ? paged_attn_tc_kernel<true, false> : paged_attn_tc_kernel<false, false>, g, b, kPtSmem, s, true,
                  static_cast<PaParams&>(p));
}

}  // namespace tss
