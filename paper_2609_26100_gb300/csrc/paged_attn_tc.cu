// Attention of wide draft blocks over the paged 4-bit cache on the 5th-generation tensor cores (tcgen05),
// head_dim 128: the operation of paged_attn.cu for more than kPaTcRows query rows of a KV head (trees, long
// chains, grouped heads), which take the MMA's 128-row side.  Per page of 64 tokens, g a group of 64 dims:
//   S_g [128 rows x 64 keys] = Q_g C_g^T            score = f (s_0 S_0 + s_1 S_1 + z_0 q_0 + z_1 q_1)
//   O_g [128 rows x 64 dims] += (P s'_g) C'_g       o = (2^24 O_g + sum_t p_t z'_tg) / sum_t p_t
// C, C' are the codes as fp16 subnormals (paged_attn.cu); scales, minima, references and sums are fp32,
// Q exact in fp16 (scaled by a power of two), the weights two fp16 parts.
//
// A nibble word (8 dims of a key, or 8 keys of a dim) becomes one 16-byte chunk of a K-major operand by four
// ANDs and a shift; the order of the 8 within it (0, 4, 1, 5, 2, 6, 3, 7) and the factor 16 of odd nibbles are
// matched in Q and P.
//
// Roles (448 threads): warp 0 copies pages (one bulk copy each), warp 1 issues MMAs, warps 2-5 expand codes
// and parameters, warps 6-13 are the softmax: thread = (row, 32 of the 64 keys).  Two buffers of operands and
// scores, so that a page's expansion and scores run under the softmax before it.  Runs of pages as in
// paged_attn.cu, one CTA an SM; partials of shared items are joined by the last CTA in CTA order.
// Every wait is bounded; on expiry the kernel records a timeout, drains its copies and MMAs and returns.
#include <cstddef>

#include "paged_attn.cuh"

namespace tss {
namespace {

constexpr int kPtD = 128, kPtRows = 128, kPtKeys = 64;
constexpr int kPtThreads = 448, kPtSoft = 256;    // threads; those of the softmax
constexpr int kPtRaw = 4;                         // pages in the ring of copies
using PtBlock = PgBlock<kPtD>;
constexpr int kPtQ = kPtRows * 64 * 2;            // one group of Q: 128 rows of 128 bytes
constexpr int kPtOp = kPtKeys * 64 * 2;           // one group of C or C': 64 rows of 128 bytes
constexpr int kPtP = kPtRows * kPtKeys * 2;       // one part of one group's weights
constexpr int kPtParams = 9;                      // arrays of 64: s0 s1 z0 z1 of K, the same of V, log2 of V's larger scale
constexpr uint32_t kPtTmem = 512;                 // S: 2 buffers x 2 groups x 64 columns; O: 128 from column 256

struct __align__(16) PtShared {
  float par[2][kPtParams][kPtKeys];                   // (read as 16-byte vectors)
  uint64_t raw_full[kPtRaw], raw_free[kPtRaw], kv_full[2], kv_free[2], s_full[2], s_free[2], p_full, p_free, q_full, o_full, drain;
  uint32_t tmem;
  int abort, last, bad[kPtRaw], bad_kv[2];
  float f[kPtRows], zq[2][kPtRows], top[2][kPtRows];  // per row: factor of the scores, query sums; maxima of its halves
  float part[2][3][kPtRows];                          // the halves' sums: p, p z'_0, p z'_1
};
static_assert(offsetof(PtShared, par) % 16 == 0 && offsetof(PtShared, raw_full) % 8 == 0, "alignment of vectors and barriers");
constexpr size_t kPtSmem = 1024 + 2 * kPtQ + 2 * 4 * kPtOp + 4 * kPtP + kPtRaw * PtBlock::kBytes;

__host__ __device__ constexpr uint32_t idesc_f16_m128(int n) {
  return (1u << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(128 >> 4) << 24);
}

// A word's eight codes as fp16 subnormals.
__device__ __forceinline__ uint4 expand(uint32_t x) {
  const uint32_t y = x >> 8;
  return make_uint4(x & 0x000f000fu, x & 0x00f000f0u, y & 0x000f000fu, y & 0x00f000f0u);
}

// 32 columns of a thread's TMEM lane, left in flight: tmem_wait() before they are used.
__device__ __forceinline__ void tmem_ld32_start(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// OR of v over the 64 threads of named barrier id.
__device__ __forceinline__ bool pair_or(int id, bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %1, 0;\n\t"
      "bar.red.or.pred p, %2, 64, q;\n\t"
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

__global__ void __launch_bounds__(kPtThreads, 1) paged_attn_tc_kernel(const __grid_constant__ PaParams p) {
  extern __shared__ uint8_t pt_dyn[];
  __shared__ PtShared sh;
  const uint32_t skew = (1024 - (smem_u32(pt_dyn) & 1023)) & 1023;
  uint8_t* sq = pt_dyn + skew;        // Q: group 0, group 1
  uint8_t* skv = sq + 2 * kPtQ;       // [buffer] C_0, C_1, C'_0, C'_1
  uint8_t* sp = skv + 2 * 4 * kPtOp;  // P s'_0 (first part, rest), P s'_1 (first part, rest)
  uint8_t* raw = sp + 4 * kPtP;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const PgAttnArgs& a = p.a;
  const int gq = a.hq / a.hk;
  int u0, u1, first_cta, splits;
  cta_run(p, &u0, &u1, &first_cta, &splits);
  if (tid == 0) {
    for (int i = 0; i < kPtRaw; ++i) {
      mbar_init(&sh.raw_full[i], 1);
      mbar_init(&sh.raw_free[i], 4);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.kv_full[i], 4);
      mbar_init(&sh.kv_free[i], 1);
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.s_free[i], 8);
    }
    mbar_init(&sh.p_full, 8);
    mbar_init(&sh.p_free, 1);
    mbar_init(&sh.q_full, 8);
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
        ok = __all_sync(0xffffffffu, t < kPtRaw || mbar_wait(&sh.raw_free[s], ((t / kPtRaw) - 1) & 1, abort, a.status));
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
    // ---------------- MMAs: S(t), then O += P(t - 1) C'(t - 1) ----------------
    if (lane == 0) {
      constexpr uint32_t id = idesc_f16_m128(64);
      const uint32_t q_a = smem_u32(sq), kv_a = smem_u32(skv), p_a = smem_u32(sp);
      bool ok = true;
      for (int t = 0, seg = 0; t < n && ok; ++seg) {
        const PaReq& r = p.r[request_of(u0 + t)];
        const int len = min(n - t, r.units - (u0 + t - r.off) % r.units);
        ok = mbar_wait(&sh.q_full, seg & 1, abort, a.status);
        for (int j = 0; ok && j <= len; ++j) {
          if (j < len) {
            const int u = t + j, s = u & 1;
            if (!mbar_wait(&sh.kv_full[s], (u >> 1) & 1, abort, a.status) ||
                (u >= 2 && !mbar_wait(&sh.s_free[s], ((u >> 1) - 1) & 1, abort, a.status))) {
              ok = false;
              break;
            }
            tc_fence_after();
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                umma_bf16(tm + s * 128 + g * 64, sdesc_sw128(q_a + g * kPtQ + k * 32), sdesc_sw128(kv_a + (s * 4 + g) * kPtOp + k * 32), id,
                          k ? 1u : 0u);
            umma_commit(&sh.s_full[s]);
          }
          if (j >= 1) {
            const int u = t + j - 1, s = u & 1;
            if (!mbar_wait(&sh.p_full, u & 1, abort, a.status)) {
              ok = false;
              break;
            }
            tc_fence_after();
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
              for (int part = 0; part < 2; ++part)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  umma_bf16(tm + 256 + g * 64, sdesc_sw128(p_a + (g * 2 + part) * kPtP + k * 32),
                            sdesc_sw128(kv_a + (s * 4 + 2 + g) * kPtOp + k * 32), id, (j > 1 || part || k) ? 1u : 0u);
            umma_commit(&sh.p_free);
            umma_commit(&sh.kv_free[s]);
            if (j == len) umma_commit(&sh.o_full);
          }
        }
        t += len;
      }
      // every MMA issued has completed before the kernel returns
      umma_commit(&sh.drain);
      mbar_drain(&sh.drain, 0);
    }
  } else if (warp < 6) {
    // ---------------- codes to operands, parameters to fp32 ----------------
    const int x = tid - 64;
    for (int t = 0; t < n; ++t) {
      const int s = t & 1, rs = t % kPtRaw;
      const bool ok = mbar_wait(&sh.raw_full[rs], (t / kPtRaw) & 1, abort, a.status) &&
                      (t < 2 || mbar_wait(&sh.kv_free[s], ((t >> 1) - 1) & 1, abort, a.status));
      if (!__all_sync(0xffffffffu, ok)) break;
      const uint8_t* blk = raw + rs * PtBlock::kBytes;
      const bool bad = sh.bad[rs];
      uint8_t* op = skv + s * 4 * kPtOp;
      // (without a page: zeros, so that no weight meets a stale operand)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int w = i * 128 + x;
        const uint4 zero = make_uint4(0, 0, 0, 0);
        const uint4 k = bad ? zero : *reinterpret_cast<const uint4*>(blk + PtBlock::kK + w * 16);
        const uint4 v = bad ? zero : *reinterpret_cast<const uint4*>(blk + PtBlock::kV + w * 16);
        // K: key w / 4, dims 16 (w % 4) .. + 15 of each group
        const int key = w >> 2, c = 2 * (w & 3);
        uint8_t* kd = op + key * 128;
        *reinterpret_cast<uint4*>(kd + ((c ^ (key & 7)) << 4)) = expand(k.x);
        *reinterpret_cast<uint4*>(kd + (((c + 1) ^ (key & 7)) << 4)) = expand(k.y);
        *reinterpret_cast<uint4*>(kd + kPtOp + ((c ^ (key & 7)) << 4)) = expand(k.z);
        *reinterpret_cast<uint4*>(kd + kPtOp + (((c + 1) ^ (key & 7)) << 4)) = expand(k.w);
        // V: half i, dims 4 (x / 4) .. + 3, tokens 8 b + 2 (x % 4) + i of the half
        const int d0 = (x >> 2) * 4, vc = i * 4 + (x & 3);
        uint8_t* vd = op + (2 + d0 / 64) * kPtOp + (d0 % 64) * 128;
        const uint32_t vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) *reinterpret_cast<uint4*>(vd + e * 128 + ((vc ^ ((d0 + e) & 7)) << 4)) = expand(vw[e]);
      }
      if (x < kPtKeys) {
        const __half2* kp = reinterpret_cast<const __half2*>(blk + PtBlock::kKParams) + 2 * x;
        const __half2* vp = reinterpret_cast<const __half2*>(blk + PtBlock::kVParams) + 2 * x;
        const float2 k0 = __half22float2(kp[0]), k1 = __half22float2(kp[1]), v0 = __half22float2(vp[0]), v1 = __half22float2(vp[1]);
        const float all[kPtParams] = {k0.x, k1.x, k0.y, k1.y, v0.x, v1.x, v0.y, v1.y, __log2f(fmaxf(fmaxf(v0.x, v1.x), kLeast))};
#pragma unroll
        for (int i = 0; i < kPtParams; ++i) sh.par[s][i][x] = all[i];
        if (x == 0) sh.bad_kv[s] = bad;
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&sh.kv_full[s]);
        mbar_arrive(&sh.raw_free[rs]);
      }
    }
  } else {
    // ---------------- softmax: thread = (row, half of a page's keys) ----------------
    // After a wait that gave up the threads go on without waiting, through the same barriers.
    const int sw = warp - 6, qd = warp & 3, half = sw >> 2, row = qd * 32 + lane, pair = 1 + qd;
    const uint32_t lanes = static_cast<uint32_t>(qd * 32) << 16;
    bool ok = true;
    for (int t = 0, seg = 0; t < n; ++seg) {
      const PaReq& r = p.r[request_of(u0 + t)];
      const int v = u0 + t - r.off, item = v / r.units, x0 = v - item * r.units, len = min(n - t, r.units - x0);
      const int h = item % a.hk, row0 = item / a.hk * kPtRows, rows = min(kPtRows, r.n * gq - row0);
      // Q: 16 lanes a row, 8 dims each, as chunks in the operand's order
#pragma unroll 2
      for (int i = 0; i < 8; ++i) {
        const int qr = sw * 16 + i * 2 + (lane >> 4), c8 = lane & 15;
        float x[8];
        if (qr < rows) {
          const int q = row0 + qr;
          const long long at = (r.row + q / gq) * a.qs + static_cast<long long>(h * gq + q % gq) * kPtD + c8 * 8;
          if (a.is_half)
            load_vec<__half, 8>(static_cast<const __half*>(a.q) + at, x);
          else
            load_vec<__nv_bfloat16, 8>(static_cast<const __nv_bfloat16*>(a.q) + at, x);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = 0.f;
        }
        float big = 0.f, sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          big = fmaxf(big, fabsf(x[e]));
          sum += x[e];
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
      const float2 f2 = make_float2(f, f), zq0 = make_float2(sh.zq[0][row], sh.zq[0][row]), zq1 = make_float2(sh.zq[1][row], sh.zq[1][row]);
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
      float ref = -INFINITY;
      float2 l2 = make_float2(0.f, 0.f), oz0 = l2, oz1 = l2;
      for (int j = 0; j < len; ++j) {
        const int u = t + j, s = u & 1;
        ok = __all_sync(0xffffffffu, ok && mbar_wait(&sh.kv_full[s], (u >> 1) & 1, abort, a.status) &&
                                         mbar_wait(&sh.s_full[s], (u >> 1) & 1, abort, a.status));
        tc_fence_after();
        if (active) {
          const int x = x0 + j, key0 = (x < r.sink ? x : x - r.sink + r.lo) * kPtKeys;
          uint32_t vis = 0xffffffffu;
          if (valid) vis = sh.bad_kv[s] ? 0u : static_cast<uint32_t>(row_sees(a, r, qp, anc_lo, anc_hi, key0) >> (32 * half));
          const bool all = __all_sync(0xffffffffu, vis == 0xffffffffu);
          uint32_t s0[32], s1[32];
          __syncwarp();
          tmem_ld32_start(tm + lanes + s * 128 + half * 32, s0);
          tmem_ld32_start(tm + lanes + s * 128 + 64 + half * 32, s1);
          tmem_wait();
          const float(*par)[kPtKeys] = sh.par[s];
          // scores / f, over s0
          float top = -INFINITY;
#pragma unroll
          for (int k = 0; k < 32; k += 4) {
            const float4 a0 = *reinterpret_cast<const float4*>(&par[0][half * 32 + k]), a1 = *reinterpret_cast<const float4*>(&par[1][half * 32 + k]);
            const float4 b0 = *reinterpret_cast<const float4*>(&par[2][half * 32 + k]), b1 = *reinterpret_cast<const float4*>(&par[3][half * 32 + k]);
            const float4 lg = *reinterpret_cast<const float4*>(&par[8][half * 32 + k]);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              float2 c = mul2(y ? make_float2(b0.z, b0.w) : make_float2(b0.x, b0.y), zq0);
              c = fma2(y ? make_float2(b1.z, b1.w) : make_float2(b1.x, b1.y), zq1, c);
              c = fma2(y ? make_float2(a0.z, a0.w) : make_float2(a0.x, a0.y),
                       make_float2(__uint_as_float(s0[k + 2 * y]), __uint_as_float(s0[k + 2 * y + 1])), c);
              c = fma2(y ? make_float2(a1.z, a1.w) : make_float2(a1.x, a1.y),
                       make_float2(__uint_as_float(s1[k + 2 * y]), __uint_as_float(s1[k + 2 * y + 1])), c);
              const float2 e = fma2(c, f2, y ? make_float2(lg.z, lg.w) : make_float2(lg.x, lg.y));
              if (all || (vis >> (k + 2 * y) & 1u)) top = fmaxf(top, e.x);
              if (all || (vis >> (k + 2 * y + 1) & 1u)) top = fmaxf(top, e.y);
              s0[k + 2 * y] = __float_as_uint(c.x);
              s0[k + 2 * y + 1] = __float_as_uint(c.y);
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.s_free[s]);
          // the row's reference rises where a weight times its value's scale would pass 2^15, to leave it at 2^7
          if (pair_or(pair, top - ref > 15.f)) {
            sh.top[half][row] = top;
            named_bar_sync(pair, 64);
            top = fmaxf(sh.top[0][row], sh.top[1][row]);
            float al = 1.f;
            if (top - ref > 15.f) {
              const float now = top - 7.f;
              al = ref == -INFINITY ? 1.f : ex2(ref - now);
              ref = now;
              l2 = mul2(l2, make_float2(al, al));
              oz0 = mul2(oz0, make_float2(al, al));
              oz1 = mul2(oz1, make_float2(al, al));
            }
            if (j > 0 && __any_sync(0xffffffffu, al != 1.f)) {
              ok = __all_sync(0xffffffffu, ok && mbar_wait(&sh.p_free, (u - 1) & 1, abort, a.status));
              tc_fence_after();
              __syncwarp();
              float o[16];
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                const uint32_t at = tm + lanes + 256 + half * 64 + c * 16;
                tmem_ld16(at, o);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] *= al;
                tmem_st16(at, o);
              }
              tc_fence_before();
            }
          }
          if (u > 0) ok = __all_sync(0xffffffffu, ok && mbar_wait(&sh.p_free, (u - 1) & 1, abort, a.status));
          // weights: chunk c of the row's P holds, at 2 b + i, key 8 b + 2 c + i of the half
          const float2 nref = make_float2(-ref, -ref);
          uint8_t* pd = sp + row * 128;
#pragma unroll
          for (int hc = 0; hc < 2; ++hc) {
            uint32_t hi[2][2][4], lo[2][2][4];  // [group][chunk 2 hc + y][b]
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              const int k = 8 * b + 4 * hc;
              const float4 v0 = *reinterpret_cast<const float4*>(&par[4][half * 32 + k]), v1 = *reinterpret_cast<const float4*>(&par[5][half * 32 + k]);
              const float4 w0 = *reinterpret_cast<const float4*>(&par[6][half * 32 + k]), w1 = *reinterpret_cast<const float4*>(&par[7][half * 32 + k]);
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const int kk = k + 2 * y;
                const float2 e = fma2(make_float2(__uint_as_float(s0[kk]), __uint_as_float(s0[kk + 1])), f2, nref);
                float2 w = make_float2(ex2(e.x), ex2(e.y));
                const float2 z0 = y ? make_float2(w0.z, w0.w) : make_float2(w0.x, w0.y), z1 = y ? make_float2(w1.z, w1.w) : make_float2(w1.x, w1.y);
                const float2 c0 = y ? make_float2(v0.z, v0.w) : make_float2(v0.x, v0.y), c1 = y ? make_float2(v1.z, v1.w) : make_float2(v1.x, v1.y);
                float2 p0, p1;
                const float2 down = make_float2(0.0625f, 0.0625f);  // (odd nibbles stand four bits up)
                if (all) {
                  l2 = add2(l2, w);
                  oz0 = fma2(w, z0, oz0);
                  oz1 = fma2(w, z1, oz1);
                  if (b & 1) w = mul2(w, down);
                  p0 = mul2(w, c0);
                  p1 = mul2(w, c1);
                } else {  // (what the row does not see may be NaN: selected away, not multiplied)
                  const bool on0 = vis >> kk & 1u, on1 = vis >> (kk + 1) & 1u;
                  w = make_float2(on0 ? w.x : 0.f, on1 ? w.y : 0.f);
                  l2 = add2(l2, w);
                  oz0 = fma2(w, make_float2(on0 ? z0.x : 0.f, on1 ? z0.y : 0.f), oz0);
                  oz1 = fma2(w, make_float2(on0 ? z1.x : 0.f, on1 ? z1.y : 0.f), oz1);
                  if (b & 1) w = mul2(w, down);
                  p0 = make_float2(on0 ? w.x * c0.x : 0.f, on1 ? w.y * c0.y : 0.f);
                  p1 = make_float2(on0 ? w.x * c1.x : 0.f, on1 ? w.y * c1.y : 0.f);
                }
                const float2 minus = make_float2(-1.f, -1.f);
                hi[0][y][b] = pack_f16(p0.x, p0.y);
                hi[1][y][b] = pack_f16(p1.x, p1.y);
                const float2 r0 = fma2(__half22float2(*reinterpret_cast<const __half2*>(&hi[0][y][b])), minus, p0);
                const float2 r1 = fma2(__half22float2(*reinterpret_cast<const __half2*>(&hi[1][y][b])), minus, p1);
                lo[0][y][b] = pack_f16(r0.x, r0.y);
                lo[1][y][b] = pack_f16(r1.x, r1.y);
              }
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int at = ((half * 4 + 2 * hc + y) ^ (row & 7)) << 4;
#pragma unroll
              for (int g = 0; g < 2; ++g) {
                *reinterpret_cast<uint4*>(pd + (2 * g) * kPtP + at) = make_uint4(hi[g][y][0], hi[g][y][1], hi[g][y][2], hi[g][y][3]);
                *reinterpret_cast<uint4*>(pd + (2 * g + 1) * kPtP + at) = make_uint4(lo[g][y][0], lo[g][y][1], lo[g][y][2], lo[g][y][3]);
              }
            }
          }
          fence_async_smem();
        } else {  // no row of the quadrant is in use: the arrivals alone, in step with the others
          if (u > 0) ok = __all_sync(0xffffffffu, ok && mbar_wait(&sh.p_free, (u - 1) & 1, abort, a.status));
          if (lane == 0) mbar_arrive(&sh.s_free[s]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full);
      }
      // ---- the segment's end ----
      ok = __all_sync(0xffffffffu, ok && mbar_wait(&sh.o_full, seg & 1, abort, a.status));
      tc_fence_after();
      const bool whole = x0 == 0 && len == r.units;
      int c0 = first_cta, c1 = first_cta + splits - 1;
      if (!whole && !p.aligned) {
        c0 = cta_of_unit(u0 + t - x0, p.total);
        c1 = cta_of_unit(u0 + t - x0 + r.units - 1, p.total);
      }
      if (active) {
        sh.part[half][0][row] = l2.x + l2.y;
        sh.part[half][1][row] = oz0.x + oz0.y;
        sh.part[half][2][row] = oz1.x + oz1.y;
        named_bar_sync(pair, 64);
        const float L = sh.part[0][0][row] + sh.part[1][0][row], z = sh.part[0][1 + half][row] + sh.part[1][1 + half][row];
        const long long slot = (blockIdx.x * 2 + (x0 == 0 ? 1 : 0)) * static_cast<long long>(kPtRows) + row;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          float o[16];
          __syncwarp();
          tmem_ld16(tm + lanes + 256 + half * 64 + c * 16, o);
          if (!valid) continue;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 x = make_float4(fmaf(o[4 * i], 16777216.f, z), fmaf(o[4 * i + 1], 16777216.f, z), fmaf(o[4 * i + 2], 16777216.f, z),
                                         fmaf(o[4 * i + 3], 16777216.f, z));
            const int c4 = half * 16 + c * 4 + i;
            if (whole)
              finish_row<kPtD>(a, r, h, row0 + row, c4, ref, L, x);
            else
              __stcg(reinterpret_cast<float4*>(p.part_o + slot * kPtD) + c4, x);
          }
        }
        if (!whole && valid && half == 0) __stcg(p.part_ml + slot, make_float2(ref, L));
        tc_fence_before();
      }
      named_bar_sync(5, kPtSoft);
      if (!whole) {
        if (sw == 0 && lane == 0) {
          sh.last = atom_add_acq_rel_gpu(&p.counters[c0], 1) == c1 - c0;
          if (sh.last) atomicExch(&p.counters[c0], 0);
        }
        named_bar_sync(5, kPtSoft);
        if (sh.last)
          for (int q = sw; q < rows; q += 8) {
            float M, L;
            float4 x;
            gather_partials<kPtD>(p, kPtRows, c0, c1, q, 0, 1, &M, &L, &x);
            finish_row<kPtD>(a, r, h, row0 + q, lane, M, L, x);
          }
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
  return cudaFuncSetAttribute(paged_attn_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kPtSmem));
}

cudaError_t launch_paged_attention_tc(PaParams& p, int sms, cudaStream_t s) {
  // (two pages at least, so that the copy, the expansion and the scores of one run under the other's softmax; an
  // item's start and end cost about as much as 6)
  const int grid = pa_cut(p, sms, 2, 6);
  return launch_k(paged_attn_tc_kernel, dim3(grid), dim3(kPtThreads), kPtSmem, s, true, p);
}

}  // namespace tss
