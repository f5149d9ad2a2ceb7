// Attention of wide draft blocks over the paged 4-bit cache on the 5th-generation tensor cores (tcgen05),
// head_dim 128: the operation of paged_attn.cu for more than kPaTcRows query rows of a KV head (trees, long
// chains, grouped heads), which take the MMA's 128-row side.  Per page of 64 tokens, g a group of 64 dims:
//   S_g [128 rows x 64 keys] = Q_g C_g^T            score = f (s_0 S_0 + s_1 S_1 + z_0 q_0 + z_1 q_1)
//   O_g [128 rows x 64 dims] += (P s'_g) C'_g       o = (2^24 O_g + sum_t p_t z'_tg) / sum_t p_t
// C, C' are the codes as fp16 subnormals (paged_attn.cu); scales, minima, references and sums are fp32,
// Q exact in fp16 (scaled by a power of two), the weights one fp16 part (bf16 outputs) or two.
//
// A nibble word (8 dims of a key, or 8 keys of a dim) becomes one 16-byte chunk of a K-major operand by four
// ANDs and a shift; the order of the 8 within it (0, 4, 1, 5, 2, 6, 3, 7) and the factor 16 of odd nibbles are
// matched in Q and P.
//
// Roles (640 threads): warp 0 copies pages (one bulk copy each), warp 1 issues MMAs, warps 2-3 expand codes
// and parameters, warps 4-19 are the softmax: thread = (row, 16 of the 64 keys).  Two buffers of operands, three
// of scores: a page's expansion and scores run under the softmax of the pages before it.  Runs of pages as in
// paged_attn.cu, one CTA an SM; partials of shared items are joined by the last CTA in CTA order.
// Every wait is bounded; on expiry the kernel records a timeout, drains its copies and MMAs and returns.
//
// Bound: the softmax, 1.7 us a page of 64 keys and 128 rows, of which about 1.2 us are its reads of the keys' parameters from
// shared memory (nine floats a key, the same for every row, at 128 bytes a clock); the MMAs take 0.3 us of it.  About
// 20 us more a launch: first page, start and end of an item.  128 rows, 32 heads, four requests of 4600 tokens 137 us.
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
constexpr int kPtP = kPtRows * kPtKeys * 2;       // one part of one group's weights
constexpr int kPtParams = 9;                      // arrays of 64: s0 s1 z0 z1 of K, the same of V, log2 of V's larger scale
constexpr uint32_t kPtTmem = 512;                 // S: 3 buffers x 2 groups x 64 columns; O: 128 from column kPtO
constexpr uint32_t kPtO = 384;

struct __align__(16) PtShared {
  float par[4][kPtParams][kPtKeys];                   // (read as 16-byte vectors)
  uint64_t raw_full[kPtRaw], raw_free[kPtRaw], k_full[2], k_free[2], v_full[2], v_free[2], s_full[3], s_free[3], p_full[2], p_free[2], par_full[4], q_full, o_full, drain;
  uint32_t tmem;
  int abort, last, bad[kPtRaw], bad_par[4];
  float f[kPtRows], zq[2][kPtRows], top[4][kPtRows];  // per row: factor of the scores, query sums; maxima of its quarters
  float part[4][3][kPtRows];                          // the quarters' sums: p, p z'_0, p z'_1
};
static_assert(offsetof(PtShared, par) % 16 == 0 && offsetof(PtShared, raw_full) % 8 == 0, "alignment of vectors and barriers");
constexpr size_t kPtSmem = 1024 + 2 * kPtQ + 2 * 4 * kPtOp + 4 * kPtP + kPtRaw * PtBlock::kBytes;

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

// 16 columns of a thread's TMEM lane, left in flight: tmem_wait() before they are used.
__device__ __forceinline__ void tmem_ld16_start(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

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
__device__ __forceinline__ unsigned long long row_sees(const PgAttnArgs& a, const PaReq& r, int qp, unsigned long long lo, unsigned long long hi,
                                                       int key0) {
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
    const int from = qp - a.window + 1 - key0, sinks = a.sinks - key0;
    unsigned long long near = from <= 0 ? ~0ull : from >= 64 ? 0ull : ~0ull << from;
    if (a.positions && blk) {  // a row of the block stands at its own position
      near &= ~blk;
      for (unsigned long long x = v & blk; x; x &= x - 1) {
        const int i = __ffsll(static_cast<long long>(x)) - 1;
        if (qp - max(__ldg(a.positions + r.row + key0 + i - r.first), r.first) < a.window) near |= 1ull << i;
      }
    }
    v &= near | (sinks >= 64 ? ~0ull : sinks <= 0 ? 0ull : (1ull << sinks) - 1);
  }
  return v;
}

// The softmax team of an item's last CTA joins the partials of CTAs c0..c1: first every row's weights of them (in
// P's and Q's shared memory: no MMA is in flight), then 4 dims of 8 rows a thread, their loads in flight together.
__device__ __forceinline__ void join_parts(const PaParams& p, PtShared& sh, uint8_t* sq, uint8_t* sp, const PaReq& r, int h, int row0, int rows,
                                           int c0, int c1, int sw, int qt, int row, int lane) {
  const int parts = c1 - c0 + 1;
  constexpr int kFirst = 4 * kPtP / (kPtRows * 4);  // weights that P's memory takes: 128 partials
  const auto weight = [&](int x) {
    return (x < kFirst ? reinterpret_cast<float*>(sp) + x * kPtRows : reinterpret_cast<float*>(sq) + (x - kFirst) * kPtRows);
  };
  const auto slot = [&](int x) { return static_cast<long long>((c0 + x) * 2 + (x == 0)) * kPtRows; };
  float M = -INFINITY, L = 0.f;
  if (row < rows)
#pragma unroll 4
    for (int x = qt; x < parts; x += 4) M = fmaxf(M, __ldcg(p.part_ml + slot(x) + row).x);
  sh.top[qt][row] = M;
  named_bar_sync(5, kPtSoft);
  M = fmaxf(fmaxf(sh.top[0][row], sh.top[1][row]), fmaxf(sh.top[2][row], sh.top[3][row]));
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
#pragma unroll
  for (int i = 0; i < kRowsOf; ++i) {
    const int q = sw + i * kPtSoftWarps;
    if (q >= rows) continue;
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m = fmaxf(m, sh.top[k][q]);
      l += sh.part[k][0][q];
    }
    finish_row<kPtD>(p.a, r, h, row0 + q, lane, m, l, o[i]);
  }
}

// TWO: weights of two fp16 parts (fp16 outputs); else one (bf16 outputs: its 2^-12 is a fraction of their own 2^-9),
// and then two buffers of them.
template <bool TWO>
__global__ void __launch_bounds__(kPtThreads, 1) paged_attn_tc_kernel(const __grid_constant__ PaParams p) {
  extern __shared__ uint8_t pt_dyn[];
  __shared__ PtShared sh;
  const uint32_t skew = (1024 - (smem_u32(pt_dyn) & 1023)) & 1023;
  uint8_t* sq = pt_dyn + skew;        // Q: group 0, group 1
  uint8_t* skv = sq + 2 * kPtQ;       // [buffer] C_0, C_1, C'_0, C'_1
  uint8_t* sp = skv + 2 * 4 * kPtOp;  // P s'_0, P s'_1; then their second parts, or the same of the other buffer
  uint8_t* raw = sp + 4 * kPtP;
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
      mbar_init(&sh.p_full[i], kPtSoftWarps);
      mbar_init(&sh.p_free[i], 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(&sh.par_full[i], kPtExpand);
    for (int i = 0; i < 3; ++i) {
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.s_free[i], kPtSoftWarps);
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
  griddep_wait();
  griddep_launch();
  const uint32_t tm = sh.tmem;
  volatile int* abort = &sh.abort;
  const int n = u1 - u0;  // pages of the run; page t of it is unit u0 + t
  // P's buffer of page u, and the parity of its barriers' phases: two buffers of one part or one of two parts
  const auto p_buf = [](int u) { return TWO ? 0 : u & 1; };
  const auto p_par = [](int u) { return static_cast<uint32_t>(TWO ? u & 1 : (u >> 1) & 1); };
  constexpr int kPBufs = TWO ? 1 : 2;
  constexpr int kPBuf = TWO ? 4 * kPtP : 2 * kPtP;
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
      long long blk = -1;
      if (t0 + lane < n) {
        const int u = u0 + t0 + lane;
        const PaReq& r = p.r[request_of(u)];
        const int v = u - r.off, item = v / r.units, x = v - item * r.units, at = x < r.sink ? x : x - r.sink + r.lo;
        const int page = __ldg(a.table + static_cast<long long>(r.seq) * a.max_pages + at);
        if (page >= 0 && page < a.n_pages)
          blk = static_cast<long long>(page) * a.hk + item % a.hk;
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
    if (lane == 0) {
      constexpr uint32_t id = idesc_f16_m128(64);
      const uint32_t q_a = smem_u32(sq), kv_a = smem_u32(skv), p_a = smem_u32(sp);
      bool ok = true;
      for (int t = 0, seg = 0; t < n && ok; ++seg) {
        const PaReq& r = p.r[request_of(u0 + t)];
        const int len = min(n - t, r.units - (u0 + t - r.off) % r.units);
        const auto scores = [&](int u) {
          const int s = u & 1, b = u % 3;
          if (!mbar_wait(&sh.k_full[s], (u >> 1) & 1, abort, a.status) ||
              (u >= 3 && !mbar_wait(&sh.s_free[b], (u / 3 - 1) & 1, abort, a.status)))
            return false;
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
          const int u = t + j, s = u & 1;
          ok = mbar_wait(&sh.v_full[s], (u >> 1) & 1, abort, a.status) && mbar_wait(&sh.p_full[p_buf(u)], p_par(u), abort, a.status);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int part = 0; part < (TWO ? 2 : 1); ++part)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                umma_bf16(tm + kPtO + g * 64, sdesc_sw128(p_a + p_buf(u) * kPBuf + (part * 2 + g) * kPtP + k * 32),
                          sdesc_sw128(kv_a + (s * 4 + 2 + g) * kPtOp + k * 32), id, (j || part || k) ? 1u : 0u);
          umma_commit(&sh.p_free[p_buf(u)]);
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
        const uint2 kp = *reinterpret_cast<const uint2*>(blk + PtBlock::kKParams + 8 * x), vp = *reinterpret_cast<const uint2*>(blk + PtBlock::kVParams + 8 * x);
        const auto pair = [](uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); };
        const float2 k0 = pair(kp.x), k1 = pair(kp.y), v0 = pair(vp.x), v1 = pair(vp.y);
        const float all[kPtParams] = {k0.x, k1.x, k0.y, k1.y, v0.x, v1.x, v0.y, v1.y, __log2f(fmaxf(fmaxf(v0.x, v1.x), kLeast))};
#pragma unroll
        for (int i = 0; i < kPtParams; ++i) sh.par[t & 3][i][x] = all[i];
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
        // unit w: half w / 128, dims 4 (w / 4 % 32) .. + 3, tokens 8 b + 2 (w % 4) + i of the half
        const int w = i * 32 * kPtExpand + x, d0 = ((w >> 2) & 31) * 4, vc = (w >> 7) * 4 + (w & 3);
        const uint4 v = bad ? zero : *reinterpret_cast<const uint4*>(blk + PtBlock::kV + w * 16);
        uint8_t* vd = op + (2 + d0 / 64) * kPtOp + (d0 % 64) * 128;
        const uint32_t vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) *reinterpret_cast<uint4*>(vd + e * 128 + ((vc ^ ((d0 + e) & 7)) << 4)) = expand(vw[e]);
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&sh.v_full[s]);
        mbar_arrive(&sh.raw_free[rs]);
      }
    }
  } else {
    // ---------------- softmax: thread = (row, a quarter of a page's keys) ----------------
    // Quarter qt: keys 16 qt .. + 15, which are half of each of four chunks of the row's P.
    // After a wait that gave up the threads go on without waiting, through the same barriers.
    const int sw = warp - 2 - kPtExpand, qd = warp & 3, qt = sw >> 2, half = qt >> 1;
    const int row = qd * 32 + lane, quad = 1 + qd;
    const uint32_t lanes = static_cast<uint32_t>(qd * 32) << 16;
    bool ok = true;
    for (int t = 0, seg = 0; t < n; ++seg) {
      const int rb = request_of(u0 + t);
      const PaReq& r = p.r[rb];
      const int v = u0 + t - r.off, item = v / r.units, x0 = v - item * r.units, len = min(n - t, r.units - x0);
      const int h = item % a.hk, row0 = item / a.hk * kPtRows, rows = min(kPtRows, r.n * gq - row0);
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
        if (c8 == 0) sh.f[qr] = a.scale_log2 * 16777216.f / up;
        if ((c8 & 7) == 0) sh.zq[c8 >> 3][qr] = sum * (up * 5.9604645e-8f);
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.q_full);
      named_bar_sync(5, kPtSoft);
      const bool valid = row < rows, active = qd * 32 < rows;
      const float f = sh.f[row];
      const f2_t f2 = f2_pack(f, f), zq0 = f2_pack(sh.zq[0][row], sh.zq[0][row]), zq1 = f2_pack(sh.zq[1][row], sh.zq[1][row]);
      int qp = 0;
      unsigned long long anc_lo = ~0ull, anc_hi = ~0ull;
      if (valid) {
        const int ti = (row0 + row) / gq;
        qp = a.positions ? max(__ldg(a.positions + r.row + ti), r.first) : r.first + ti;
        if (a.mask) {
          anc_lo = __ldg(a.mask + 2LL * (r.row + ti));
          anc_hi = __ldg(a.mask + 2LL * (r.row + ti) + 1);
        } else {
          anc_lo = ti >= 63 ? ~0ull : (2ull << ti) - 1;
          anc_hi = ti < 64 ? 0ull : ti == 127 ? ~0ull : (2ull << (ti - 64)) - 1;
        }
        // (rows that the block does not have are not seen, whatever the mask says)
        if (r.n < 64) anc_lo &= (1ull << r.n) - 1;
        anc_hi = r.n <= 64 ? 0ull : r.n < 128 ? anc_hi & ((1ull << (r.n - 64)) - 1) : anc_hi;
      }
      // pages whose keys every row sees: [0, all0), the sinks', and [all1, all2)
      int pmax = 0;
      if (a.window) {
        pmax = valid ? qp : 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) pmax = max(pmax, __shfl_xor_sync(0xffffffffu, pmax, o));
      }
      const int all0 = a.window ? min(r.sink, a.sinks / kPtKeys) : 0;
      const int all1 = r.sink + (a.window ? max(0, (pmax - a.window + kPtKeys) / kPtKeys - r.lo) : 0);
      const int all2 = r.sink + r.first / kPtKeys - r.lo;
      float ref = -INFINITY;
      f2_t l2 = f2_pack(0.f, 0.f), oz0 = l2, oz1 = l2;
      for (int j = 0; j < len; ++j) {
        const int u = t + j, sb = u % 3;
        ok = ok && quiet_wait(&sh.par_full[u & 3], (u >> 2) & 1, abort, a.status) && quiet_wait(&sh.s_full[sb], (u / 3) & 1, abort, a.status);
        tc_fence_after();
        if (active) {
          const int x = x0 + j;
          uint32_t vis = 0xffffu;  // bit i: key 16 qt + i
          if (sh.bad_par[u & 3])
            vis = valid ? 0u : vis;
          else if (valid && !(x < all0 || (x >= all1 && x < all2)))
            vis = static_cast<uint32_t>(row_sees(a, r, qp, anc_lo, anc_hi, (x < r.sink ? x : x - r.sink + r.lo) * kPtKeys) >> (16 * qt)) & 0xffffu;
          const auto page = [&](auto all_tag) {
            constexpr bool kAll = decltype(all_tag)::value;  // the warp's rows see all of the thread's keys
            const float* par = &sh.par[u & 3][0][16 * qt];
            const auto pr = [&](int k, int b) { return *reinterpret_cast<const ulonglong2*>(par + k * kPtKeys + 4 * b); };
            f2_t c[8];  // scores / f of keys 2 i, 2 i + 1
            {
              uint32_t s0[16], s1[16];
              __syncwarp();
              tmem_ld16_start(tm + lanes + sb * 128 + 16 * qt, s0);
              tmem_ld16_start(tm + lanes + sb * 128 + 64 + 16 * qt, s1);
              tmem_wait();
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&sh.s_free[sb]);
#pragma unroll
              for (int b = 0; b < 4; ++b) {
                const ulonglong2 a0 = pr(0, b), a1 = pr(1, b), b0 = pr(2, b), b1 = pr(3, b);
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                  const int k = 4 * b + 2 * y;
                  const f2_t m = f2_pack(__uint_as_float(s0[k]), __uint_as_float(s0[k + 1])), z = f2_pack(__uint_as_float(s1[k]), __uint_as_float(s1[k + 1]));
                  c[k / 2] = f2_fma(y ? a1.y : a1.x, z, f2_fma(y ? a0.y : a0.x, m, f2_fma(y ? b1.y : b1.x, zq1, f2_mul(y ? b0.y : b0.x, zq0))));
                }
              }
            }
            float top = -INFINITY;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              const ulonglong2 lg = pr(8, b);
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const int k = 4 * b + 2 * y;
                const float2 e = f2_unpack(f2_fma(c[k / 2], f2, y ? lg.y : lg.x));
                if constexpr (kAll) {
                  top = fmaxf(top, fmaxf(e.x, e.y));
                } else {
                  top = fmaxf(top, vis >> k & 1u ? e.x : -INFINITY);
                  top = fmaxf(top, vis >> (k + 1) & 1u ? e.y : -INFINITY);
                }
              }
            }
            // the row's reference rises where a weight times its value's scale would pass 2^15, to leave it at 2^7
            if (quad_or(quad, top - ref > 15.f)) {
              sh.top[qt][row] = top;
              named_bar_sync(quad, 128);
              top = fmaxf(fmaxf(sh.top[0][row], sh.top[1][row]), fmaxf(sh.top[2][row], sh.top[3][row]));
              float al = 1.f;
              if (top - ref > 15.f) {
                const float now = top - 7.f;
                al = ref == -INFINITY ? 1.f : ex2(ref - now);
                ref = now;
                const f2_t al2 = f2_pack(al, al);
                l2 = f2_mul(l2, al2);
                oz0 = f2_mul(oz0, al2);
                oz1 = f2_mul(oz1, al2);
              }
              if (j > 0 && __any_sync(0xffffffffu, al != 1.f)) {
                ok = ok && quiet_wait(&sh.p_free[p_buf(u - 1)], p_par(u - 1), abort, a.status);
                tc_fence_after();
                __syncwarp();
                float o[16];
#pragma unroll
                for (int x2 = 0; x2 < 2; ++x2) {
                  const uint32_t at = tm + lanes + kPtO + qt * 32 + x2 * 16;
                  tmem_ld16(at, o);
#pragma unroll
                  for (int i = 0; i < 16; ++i) o[i] *= al;
                  tmem_st16(at, o);
                }
                tc_fence_before();
              }
            }
            if (u >= kPBufs) ok = ok && quiet_wait(&sh.p_free[p_buf(u)], p_par(u - kPBufs), abort, a.status);
            // weights: chunk x of a half of the row's P holds, at 2 b + i, key 8 b + 2 x + i; b is 2 (qt & 1) + bb here
            const f2_t nref = f2_pack(-ref, -ref);
            uint8_t* pd = sp + p_buf(u) * kPBuf + row * 128 + (qt & 1) * 8;
#pragma unroll
            for (int xx = 0; xx < 2; ++xx) {  // chunks 2 xx, 2 xx + 1
              uint32_t hi[2][2][2], lo[2][2][2];  // [y: chunk 2 xx + y][group][bb]
#pragma unroll
              for (int bb = 0; bb < 2; ++bb) {
                // keys 8 bb + 4 xx + {0..3} of the quarter
                const int q4 = 2 * bb + xx;
                const ulonglong2 v0s = pr(4, q4), v1s = pr(5, q4), z0s = pr(6, q4), z1s = pr(7, q4);
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                  const int k = 4 * q4 + 2 * y;
                  const float2 e = f2_unpack(f2_fma(c[k / 2], f2, nref));
                  const float2 wf = make_float2(ex2(e.x), ex2(e.y));
                  const f2_t v0 = y ? v0s.y : v0s.x, v1 = y ? v1s.y : v1s.x, z0 = y ? z0s.y : z0s.x, z1 = y ? z1s.y : z1s.x;
                  const f2_t down = f2_pack(0.0625f, 0.0625f);  // (odd nibbles stand four bits up)
                  f2_t p0, p1;
                  if constexpr (kAll) {
                    f2_t w = f2_pack(wf.x, wf.y);
                    l2 = f2_add(l2, w);
                    oz0 = f2_fma(w, z0, oz0);
                    oz1 = f2_fma(w, z1, oz1);
                    if (bb) w = f2_mul(w, down);
                    p0 = f2_mul(w, v0);
                    p1 = f2_mul(w, v1);
                  } else {  // (what the row does not see may be NaN: selected away, not multiplied)
                    const bool on0 = vis >> k & 1u, on1 = vis >> (k + 1) & 1u;
                    const auto pick = [&](f2_t m) {
                      const float2 q = f2_unpack(m);
                      return f2_pack(on0 ? q.x : 0.f, on1 ? q.y : 0.f);
                    };
                    f2_t w = f2_pack(on0 ? wf.x : 0.f, on1 ? wf.y : 0.f);
                    l2 = f2_add(l2, w);
                    oz0 = f2_fma(w, pick(z0), oz0);
                    oz1 = f2_fma(w, pick(z1), oz1);
                    if (bb) w = f2_mul(w, down);
                    p0 = f2_mul(w, pick(v0));
                    p1 = f2_mul(w, pick(v1));
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
                  split(p0, &hi[y][0][bb], &lo[y][0][bb]);
                  split(p1, &hi[y][1][bb], &lo[y][1][bb]);
                }
              }
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const int at = ((half * 4 + 2 * xx + y) ^ (row & 7)) << 4;
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                  *reinterpret_cast<uint2*>(pd + g * kPtP + at) = make_uint2(hi[y][g][0], hi[y][g][1]);
                  if constexpr (TWO) *reinterpret_cast<uint2*>(pd + (2 + g) * kPtP + at) = make_uint2(lo[y][g][0], lo[y][g][1]);
                }
              }
            }
          };
          if (__all_sync(0xffffffffu, vis == 0xffffu))
            page(std::true_type{});
          else
            page(std::false_type{});
          fence_async_smem();
        } else {  // no row of the quadrant is in use: the arrivals alone, in step with the others
          if (u >= kPBufs) ok = ok && quiet_wait(&sh.p_free[p_buf(u)], p_par(u - kPBufs), abort, a.status);
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.s_free[sb]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full[p_buf(u)]);
      }
      // ---- the segment's end: 32 dims a thread ----
      ok = ok && quiet_wait(&sh.o_full, seg & 1, abort, a.status);
      __syncwarp();
      tc_fence_after();
      const bool whole = x0 == 0 && len == r.units;
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
        sh.part[qt][0][row] = both(l2);
        sh.part[qt][1][row] = both(oz0);
        sh.part[qt][2][row] = both(oz1);
        named_bar_sync(quad, 128);
        float L = 0.f, z = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          L += sh.part[i][0][row];
          z += sh.part[i][1 + half][row];
        }
        const long long slot = (blockIdx.x * 2 + (x0 == 0 ? 1 : 0)) * static_cast<long long>(kPtRows) + row;
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
          float o[16];
          __syncwarp();
          tmem_ld16(tm + lanes + kPtO + qt * 32 + c * 16, o);
          if (!valid) continue;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 x = make_float4(fmaf(o[4 * i], 16777216.f, z), fmaf(o[4 * i + 1], 16777216.f, z), fmaf(o[4 * i + 2], 16777216.f, z),
                                         fmaf(o[4 * i + 3], 16777216.f, z));
            const int c4 = qt * 8 + c * 4 + i;
            if (whole)
              finish_row<kPtD>(a, r, h, row0 + row, c4, ref, L, x);
            else
              __stcg(reinterpret_cast<float4*>(p.part_o + slot * kPtD) + c4, x);
          }
        }
        if (!whole && valid && qt == 0) __stcg(p.part_ml + slot, make_float2(ref, L));
        __syncwarp();
        tc_fence_before();
      }
      named_bar_sync(5, kPtSoft);
      if (!whole) {
        if (sw == 0 && lane == 0) {
          sh.last = atom_add_acq_rel_gpu(&p.counters[c0], 1) == c1 - c0;
          if (sh.last) atomicExch(&p.counters[c0], 0);
        }
        named_bar_sync(5, kPtSoft);
        if (sh.last) join_parts(p, sh, sq, sp, r, h, row0, rows, c0, c1, sw, qt, row, lane);
        named_bar_sync(5, kPtSoft);
      }
      t += len;
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tm, kPtTmem);
  }
}

}  // namespace

cudaError_t paged_attn_tc_prepare() {
  cudaError_t e = cudaFuncSetAttribute(paged_attn_tc_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kPtSmem));
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(paged_attn_tc_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kPtSmem));
  return e;
}

cudaError_t launch_paged_attention_tc(PaParams& p, int sms, cudaStream_t s) {
  // (two pages at least, so that the copy, the expansion and the scores of one run under the other's softmax; an
  // item's start and end cost about as much as 6)
  const int grid = pa_cut(p, sms, 2, 6, 6);
  return launch_k(p.a.is_half ? paged_attn_tc_kernel<true> : paged_attn_tc_kernel<false>, dim3(grid), dim3(kPtThreads), kPtSmem, s, true, p);
}

}  // namespace tss
