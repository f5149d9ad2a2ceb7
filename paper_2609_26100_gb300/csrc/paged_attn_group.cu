// Attention of the rows of many sequences over the pages that they share, on the 5th-generation tensor cores (tcgen05): the pass
// over shared keys of tss_paged_attention_shared for bf16 outputs, head_dim 128, without a window, so that every row sees every
// key.  Of a KV head and up to 128 of a group's query rows, per tile of 128 keys (two pages), g a group of 64 dims:
//   S_g [128 keys x rows] = C_g Q_g^T          e = f (s_0 S_0 + s_1 S_1) + z_0 a + z_1 b - ref,  p = 2^e
//   O [128 dims x rows] += V^T P               V = s' c' + z' in fp16, P = p in fp16
// C is K's codes as fp16 subnormals, Q exact in fp16 (paged_attn.cu); scores, references and sums of p are fp32.  The roundings
// of V and P are of 2^-12, beside the outputs' own 2^-9.
//
// Keys take the MMA's 128-row side, so a softmax thread is a key: what belongs to a key (s, z) is in its registers, what belongs to a
// row (f, a, b, ref) comes as broadcasts for two rows at a time, and the weights of eight rows leave as one vector.  In the
// orientation of paged_attn_tc.cu (a thread four rows and four keys) the latency of a page's way through a softmax warp bounds the
// kernel; here a tile's is of twice the keys, and two teams of eight warps are at different tiles (up to 64 rows) or at different
// rows of a tile (more).  A thread's sums of p are its key's; they are joined over the keys at the end.
//
// The order of a page's keys in the operands is that in which V's words hold them: a word's eight tokens are a vector of an operand
// row, and K's rows and P's follow (place 32 half + 8 t + 2 b + i of token 32 half + 8 b + 2 t + i).
//
// A row's reference is raised where a weight would pass 2^9, to where the tile's largest is at most 1: the team undoes the tile's sums,
// finds the rows' maxima, scales what it has and takes the tile again.  Values of more than 2^15 (a token whose quantised range
// passes that) enter as 2^-5 of themselves and their weights 2^5 times as large.
//
// Roles (768 threads): warp 0 copies pages, warp 1 issues MMAs, warps 2-17 are the teams (of eight warps: a quarter of the keys and
// half of the team's rows each), warps 18-19 make operands of K, 20-23 of V.  Runs of tiles
// within one item, one CTA an SM; partials of a CTA's teams are joined by the item's last CTA.  Every wait is bounded, as in
// paged_attn_tc.cu.
#include <cfloat>
#include <cstddef>
#include <type_traits>

#include "paged_attn.cuh"

namespace tss {
namespace {

constexpr int kPgrD = 128, kPgrTeam = 64, kPgrRows = 2 * kPgrTeam, kPgrKeys = 128;
constexpr int kPgrSoft = 16, kPgrMakeK = 2, kPgrMakeV = 4, kPgrThreads = 32 * (2 + kPgrSoft + kPgrMakeK + kPgrMakeV);
constexpr int kPgrRaw = 4;                      // pages in the rings of copies, of K's parts and of V's
constexpr int kPgrVals = 3;                     // pages of V's operands
constexpr int kPgrQ = kPgrTeam * 128;           // a team's rows, one group of dims
constexpr int kPgrK = kPgrKeys * 128;           // a tile's keys, one group of dims
constexpr int kPgrV = kPgrD * 128;              // 128 dims, a page's keys
constexpr int kPgrP = kPgrKeys * 128;           // a tile's keys, a team's rows
constexpr uint32_t kPgrTmem = 512, kPgrO = 256;  // S: team * 128 + group * 64; O: kPgrO + team * 64
constexpr float kPgrTop = 512.f;                // weights that raise a reference
using PgrBlock = PgBlock<kPgrD>;
constexpr int kPgrRawK = PgrBlock::kCodes + 2 * PgrBlock::kParams;  // of a page K's codes, and the parameters of K and V
constexpr int kPgrRawV = PgrBlock::kCodes + PgrBlock::kParams;      // V's codes and parameters

struct __align__(16) PgrShared {
  float4 rc[2][kPgrTeam / 2][2];                // [team][pair of rows]: f, a of both; b, -ref of both
  uint2 par[4][kPgrKeys];                       // K's (s, z) of both groups, by place; the first sign: the key's values are large
  uint64_t raw_full[2][kPgrRaw], raw_free[2][kPgrRaw], k_full[2], k_free[2], v_full[kPgrVals], v_free[kPgrVals], par_full[4], s_full[2], p_full[2], pv_done[2], q_full, drain;
  float ref[2][kPgrTeam], fac[2][kPgrTeam];
  float wmax[2][4][kPgrTeam], lsum[2][4][kPgrTeam];
  uint32_t tmem;
  int abort, last, bad_raw[2][kPgrRaw], bad[4][2];
};
static_assert(PgrBlock::kKParams + PgrBlock::kParams == PgrBlock::kVParams, "one copy brings the parameters of both");
static_assert(offsetof(PgrShared, par) % 16 == 0 && offsetof(PgrShared, raw_full) % 8 == 0, "alignment of vectors and barriers");
constexpr size_t kPgrSmem = 1024 + 4 * kPgrQ + 4 * kPgrK + kPgrVals * kPgrV + 2 * kPgrP + kPgrRaw * (kPgrRawK + kPgrRawV);

// 32 lanes x 8 columns of TMEM, left in flight until tmem_here() of the registers; stored (tmem_stored()).
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_here(uint32_t* a) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(a[0]), "+r"(a[1]), "+r"(a[2]), "+r"(a[3]), "+r"(a[4]), "+r"(a[5]), "+r"(a[6]), "+r"(a[7]));
}
__device__ __forceinline__ void tmem_here(uint32_t* a, uint32_t* b) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(a[0]), "+r"(a[1]), "+r"(a[2]), "+r"(a[3]), "+r"(a[4]), "+r"(a[5]), "+r"(a[6]), "+r"(a[7]), "+r"(b[0]), "+r"(b[1]), "+r"(b[2]),
                 "+r"(b[3]), "+r"(b[4]), "+r"(b[5]), "+r"(b[6]), "+r"(b[7]));
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n\ttcgen05.wait::st.sync.aligned;" ::"r"(taddr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// OR of v over the threads of a team's named barrier.
__device__ __forceinline__ bool team_or(int id, bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %1, 0;\n\t"
      "bar.red.or.pred p, %2, 256, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}\n"
      : "=r"(r)
      : "r"(v ? 1u : 0u), "r"(id)
      : "memory");
  return r != 0;
}
// Two pairs from shared memory.  Not volatile, so that they may be loaded ahead of stores to other places; `when` keeps them
// behind what it depends on.
__device__ __forceinline__ void pairs_at(uint32_t addr, int when, f2_t* x, f2_t* y) {
  asm("ld.shared.v2.u64 {%0, %1}, [%2];  // %3" : "=l"(*x), "=l"(*y) : "r"(addr), "r"(when));
}

// Place of a page's token among the operands' keys.
__device__ __forceinline__ int place_of(int tok) { return (tok & 33) | (tok & 6) << 2 | (tok & 24) >> 2; }

// Whether a token's values (s, z of a group) pass what fp16 weights leave room for.
__device__ __forceinline__ bool passes(uint32_t sz) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&sz));
  return fmaxf(fabsf(f.y), fabsf(fmaf(f.x, 15.f, f.y))) > 32768.f;
}
__device__ __forceinline__ __half2 h2(uint32_t x) { return *reinterpret_cast<const __half2*>(&x); }
__device__ __forceinline__ uint32_t u32(__half2 x) { return *reinterpret_cast<const uint32_t*>(&x); }

__global__ void __launch_bounds__(kPgrThreads, 1) paged_attn_group_kernel(const __grid_constant__ PaShared p) {
  extern __shared__ uint8_t pgr_dyn[];
  __shared__ PgrShared sh;
  const uint32_t skew = (1024 - (smem_u32(pgr_dyn) & 1023)) & 1023;
  uint8_t* sq = pgr_dyn + skew;      // [team][group] rows
  uint8_t* sk = sq + 4 * kPgrQ;      // [buffer][group] keys
  uint8_t* sv = sk + 4 * kPgrK;      // [page] dims
  uint8_t* sp = sv + kPgrVals * kPgrV;  // [team] keys
  uint8_t* raw_k = sp + 2 * kPgrP;
  uint8_t* raw_v = raw_k + kPgrRaw * kPgrRawK;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const PgAttnArgs& a = p.a;
  const int gq = a.hq / a.hk;
  int u0, u1, first_cta, splits;
  cta_run(p, &u0, &u1, &first_cta, &splits);
  int b = 0;
  while (b + 1 < p.n_req && p.r[b + 1].off <= u0) ++b;
  const PaReq& r = p.r[b];
  const int item = (u0 - r.off) / r.units, x0 = u0 - r.off - item * r.units, n = u1 - u0;  // n tiles of 128 keys from tile x0
  const int h = item % a.hk, row0 = item / a.hk * kPgrRows, rows = min(kPgrRows, r.n * gq - row0);
  const bool two = rows > kPgrTeam;  // the teams have rows of their own; else every second tile
  const int width0 = two ? kPgrTeam : (rows + 15) & ~15, width1 = two ? (rows - kPgrTeam + 15) & ~15 : width0;  // teams' rows, in 16s
  if (tid == 0) {
    for (int i = 0; i < kPgrRaw; ++i)
      for (int side = 0; side < 2; ++side) {
        mbar_init(&sh.raw_full[side][i], 1);
        mbar_init(&sh.raw_free[side][i], side ? kPgrMakeV : kPgrMakeK);
      }
    for (int i = 0; i < kPgrVals; ++i) {
      mbar_init(&sh.v_full[i], kPgrMakeV);
      mbar_init(&sh.v_free[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.k_full[i], kPgrMakeK);
      mbar_init(&sh.k_free[i], 1);
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.p_full[i], 1);
      mbar_init(&sh.pv_done[i], 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(&sh.par_full[i], kPgrMakeK);
    mbar_init(&sh.q_full, kPgrSoft);
    mbar_init(&sh.drain, 1);
    sh.abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&sh.tmem, kPgrTmem);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = sh.tmem;
  volatile int* abort = &sh.abort;

  if (warp == 0) {
    // ---------------- pages: K's parts and V's, each as far ahead as its ring goes (K's operands are made earlier) ----------------
    const int pages = r.first / kPgTokens, slots = 2 * n;  // (the last tile's second page may be none)
    griddep_wait();
    griddep_launch();
    int at[2] = {0, 0}, from = 0;  // parts asked for; the first page whose places the lanes hold
    const auto places = [&](int q0) {
      const int at = 2 * x0 + q0 + lane;
      if (q0 + lane >= slots || at >= pages) return -1;
      const int page = __ldcg(a.table + static_cast<long long>(r.seq) * a.max_pages + at);
      if (page >= 0 && page < a.n_pages) return page;
      report(a.status, kStatusCheck);
      return -1;
    };
    int now = places(0), later = places(32);
    uint64_t moved = globaltimer_ns();
    bool ok = true;
    while (ok && at[1] < slots) {
      bool any = false;
#pragma unroll
      for (int side = 0; side < 2; ++side) {
        const int q = at[side], s = q % kPgrRaw;
        // (K's ring is at most some pages ahead of V's, within the 64 that the lanes hold)
        if (q >= slots || q >= from + 64 || (q >= kPgrRaw && !__any_sync(0xffffffffu, mbar_test(&sh.raw_free[side][s], ((q / kPgrRaw) - 1) & 1)))) continue;
        const int page = __shfl_sync(0xffffffffu, q - from < 32 ? now : later, (q - from) & 31);
        if (lane == 0) {
          uint64_t* bar = &sh.raw_full[side][s];
          sh.bad_raw[side][s] = page < 0;
          if (page < 0) {
            mbar_arrive(bar);
          } else {
            const uint8_t* src = a.pool + (static_cast<long long>(page) * a.hk + h) * PgrBlock::kBytes;
            uint8_t* to = side ? raw_v + s * kPgrRawV : raw_k + s * kPgrRawK;
            mbar_arrive_expect_tx(bar, side ? kPgrRawV : kPgrRawK);
            bulk_load(to, src + (side ? PgrBlock::kV : PgrBlock::kK), PgrBlock::kCodes, bar);
            bulk_load(to + PgrBlock::kCodes, src + (side ? PgrBlock::kVParams : PgrBlock::kKParams), side ? PgrBlock::kParams : 2 * PgrBlock::kParams, bar);
          }
        }
        __syncwarp();
        ++at[side];
        any = true;
      }
      if (at[1] >= from + 32) {
        from += 32;
        now = later;
        later = places(from + 32);
      }
      if (any) {
        moved = globaltimer_ns();
      } else {
        __nanosleep(40);
        const bool late = globaltimer_ns() - moved > kWaitLimitNs;
        if (__any_sync(0xffffffffu, late || *abort != 0)) {
          if (lane == 0 && *abort == 0) {
            *abort = 1;
            report(a.status, kStatusTimeout);
          }
          ok = false;
        }
      }
    }
    // the copies issued last have landed before the kernel returns
    for (int side = 0; side < 2; ++side)
      for (int k = max(0, at[side] - kPgrRaw); k < at[side]; ++k) mbar_drain(&sh.raw_full[side][k % kPgrRaw], (k / kPgrRaw) & 1);
  } else if (warp == 1) {
    // ---------------- MMAs ----------------
    griddep_wait();
    griddep_launch();
    if (lane == 0) {
      const uint32_t q_a = smem_u32(sq), k_a = smem_u32(sk), v_a = smem_u32(sv), p_a = smem_u32(sp);
      constexpr uint32_t id_pv = idesc_f16_m128(kPgrTeam) | (1u << 16);  // (P: rows contiguous)
      const auto wait = [&](uint64_t* bar, int phase) { return mbar_wait(bar, phase & 1, abort, a.status); };
      const auto scores = [&](int team, int t) {
        const uint32_t id = idesc_f16_m128(team ? width1 : width0);
        const int rows_of = two ? team : 0;
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            umma_bf16(tm + team * 128 + g * 64, sdesc_sw128(k_a + ((t & 1) * 2 + g) * kPgrK + k * 32),
                      sdesc_sw128(q_a + (rows_of * 2 + g) * kPgrQ + k * 32), id, k ? 1u : 0u);
        umma_commit(&sh.s_full[team]);
      };
      const auto values = [&](int t) { return wait(&sh.v_full[2 * t % kPgrVals], 2 * t / kPgrVals) && wait(&sh.v_full[(2 * t + 1) % kPgrVals], (2 * t + 1) / kPgrVals); };
      const auto outputs = [&](int team, int t, bool first, bool last) {  // last: V's last use
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
          const int s = (2 * t + pg) % kPgrVals;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            umma_bf16(tm + kPgrO + team * 64, sdesc_sw128(v_a + s * kPgrV + k * 32), sdesc_sw128_mn(p_a + team * kPgrP + (pg * 4 + k) * 16 * 128, kPgrP),
                      id_pv, first && pg == 0 && k == 0 ? 0u : 1u);
          if (last) umma_commit(&sh.v_free[s]);
        }
        umma_commit(&sh.pv_done[team]);
      };
      bool ok = !(p.withhold && blockIdx.x == 0) && wait(&sh.q_full, 0);
      if (two) {
        ok = ok && wait(&sh.k_full[0], 0);
        if (ok) {
          tc_fence_after();
          scores(0, 0);
          scores(1, 0);
          umma_commit(&sh.k_free[0]);
        }
        for (int t = 0; t < n && ok; ++t) {
          const bool more = t + 1 < n;
          ok = values(t) && wait(&sh.p_full[0], t);
          if (!ok) break;
          tc_fence_after();
          outputs(0, t, t == 0, false);
          ok = !more || wait(&sh.k_full[(t + 1) & 1], (t + 1) >> 1);
          if (!ok) break;
          tc_fence_after();
          if (more) scores(0, t + 1);
          ok = wait(&sh.p_full[1], t);
          if (!ok) break;
          tc_fence_after();
          outputs(1, t, t == 0, true);
          if (more) {
            scores(1, t + 1);
            umma_commit(&sh.k_free[(t + 1) & 1]);
          }
        }
      } else {
        const auto tile = [&](int t) {
          if (!wait(&sh.k_full[t & 1], t >> 1)) return false;
          tc_fence_after();
          scores(t & 1, t);  // (its team's last tile but one was read out before its P was)
          umma_commit(&sh.k_free[t & 1]);
          return true;
        };
        ok = ok && tile(0) && (n < 2 || tile(1));
        for (int t = 0; t < n && ok; ++t) {
          ok = values(t) && wait(&sh.p_full[t & 1], t >> 1);
          if (!ok) break;
          tc_fence_after();
          outputs(t & 1, t, t < 2, true);
          ok = t + 2 >= n || tile(t + 2);
        }
      }
      // every MMA issued has completed before the kernel returns
      umma_commit(&sh.drain);
      mbar_drain(&sh.drain, 0);
    }
  } else if (warp >= 2 + kPgrSoft) {
    // ---------------- operands ----------------
    // A thread reads all that it needs of the pages before it stores anything, so that the loads are on their way together.
    griddep_wait();
    griddep_launch();
    const bool is_k = warp < 2 + kPgrSoft + kPgrMakeK;
    const int x = tid - 32 * (2 + kPgrSoft + (is_k ? 0 : kPgrMakeK));
    const uint4 zero = make_uint4(0, 0, 0, 0);
    if (is_k) {
      // Keys x / 4 + 16 i, dims 16 (x % 4) .. + 15 of each group; and what belongs to key x of each page, in a buffer of four
      // (S(t - 2), which is complete, was issued after the team of tile t - 4 was done).
      for (int t = 0; t < n; ++t) {
        bool here = true;
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) here = here && quiet_wait(&sh.raw_full[0][(2 * t + pg) % kPgrRaw], ((2 * t + pg) / kPgrRaw) & 1, abort, a.status);
        if (!__all_sync(0xffffffffu, here)) break;
        uint4 k[2][4];
        uint2 kp[2];
        bool bad[2];
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
          const int s = (2 * t + pg) % kPgrRaw;
          const uint8_t* blk = raw_k + s * kPgrRawK;
          bad[pg] = sh.bad_raw[0][s] != 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) k[pg][i] = *reinterpret_cast<const uint4*>(blk + (x + 64 * i) * 16);
          kp[pg] = *reinterpret_cast<const uint2*>(blk + PgrBlock::kCodes + 8 * x);
          const uint2 vp = *reinterpret_cast<const uint2*>(blk + PgrBlock::kCodes + PgrBlock::kParams + 8 * x);
          kp[pg].x = (kp[pg].x & 0xffff7fffu) | (passes(vp.x) || passes(vp.y) ? 0x8000u : 0u);  // (scales are not negative)
        }
        if (!__all_sync(0xffffffffu, t < 2 || quiet_wait(&sh.k_free[t & 1], ((t >> 1) - 1) & 1, abort, a.status))) break;
        uint8_t* op = sk + (t & 1) * 2 * kPgrK;
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
          sh.par[t & 3][pg * 64 + place_of(x)] = bad[pg] ? make_uint2(0, 0) : kp[pg];
          if (x == 0) sh.bad[t & 3][pg] = bad[pg];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int row = pg * 64 + place_of((x >> 2) + 16 * i), c = 2 * (x & 3);
            const uint4 w = bad[pg] ? zero : k[pg][i];
            uint8_t *to0 = op + row * 128 + ((c ^ (row & 7)) << 4), *to1 = op + row * 128 + (((c + 1) ^ (row & 7)) << 4);
            *reinterpret_cast<uint4*>(to0) = expand(w.x);
            *reinterpret_cast<uint4*>(to1) = expand(w.y);
            *reinterpret_cast<uint4*>(to0 + kPgrK) = expand(w.z);
            *reinterpret_cast<uint4*>(to1 + kPgrK) = expand(w.w);
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&sh.par_full[t & 3]);
          mbar_arrive(&sh.k_full[t & 1]);
          mbar_arrive(&sh.raw_free[0][(2 * t) % kPgrRaw]);
          mbar_arrive(&sh.raw_free[0][(2 * t + 1) % kPgrRaw]);
        }
      }
    } else {
      // V, a page at a time: of half a page the tokens 8 b + 2 t4 + i, a vector of a dim's row; of dims d0 .. + 3 and d0 + 32 .. + 35
      const int t4 = x & 3, half = (x >> 5) & 1, group = x >> 6, d0 = group * 64 + ((x >> 2) & 7) * 4;
      const __half2 sixteenth = __half2half2(__ushort_as_half(0x2c00)), m64 = __half2half2(__ushort_as_half(0xd400)),
                    m1024 = __half2half2(__ushort_as_half(0xe400));
      for (int q = 0; q < 2 * n; ++q) {
        const int rs = q % kPgrRaw, vs = q % kPgrVals;
        if (!__all_sync(0xffffffffu, quiet_wait(&sh.raw_full[1][rs], (q / kPgrRaw) & 1, abort, a.status))) break;
        const uint8_t* blk = raw_v + rs * kPgrRawV;
        const bool bad = sh.bad_raw[1][rs] != 0;
        uint4 v[2];
        uint2 ev[4], od[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i] = *reinterpret_cast<const uint4*>(blk + (half * 128 + (d0 / 4 + 8 * i) * 4 + t4) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          ev[i] = *reinterpret_cast<const uint2*>(blk + PgrBlock::kCodes + 8 * (32 * half + 8 * i + 2 * t4));
          od[i] = *reinterpret_cast<const uint2*>(blk + PgrBlock::kCodes + 8 * (32 * half + 8 * i + 2 * t4 + 1));
        }
        __half2 s[4], z[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t e = group ? ev[i].y : ev[i].x, o = group ? od[i].y : od[i].x;
          // (either group's values decide)
          const __half2 down = __half2half2(__ushort_as_half(0x2800));  // 2^-5
          if (passes(ev[i].x) || passes(ev[i].y)) e = u32(__hmul2(h2(e), down));
          if (passes(od[i].x) || passes(od[i].y)) o = u32(__hmul2(h2(o), down));
          s[i] = h2(__byte_perm(e, o, 0x5410));
          z[i] = h2(__byte_perm(e, o, 0x7632));
        }
        if (!__all_sync(0xffffffffu, q < kPgrVals || quiet_wait(&sh.v_free[vs], (q / kPgrVals - 1) & 1, abort, a.status))) break;
        uint8_t* op = sv + vs * kPgrV + d0 * 128;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t vw[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t lo = vw[e], hi = vw[e] >> 8;
            // codes as 1024 + c, or 1024 + 16 c from nibbles four bits up; to c exactly
            const __half2 k0 = __hadd2(h2((lo & 0x000f000fu) | 0x64006400u), m1024), k1 = __hfma2(h2((lo & 0x00f000f0u) | 0x64006400u), sixteenth, m64);
            const __half2 k2 = __hadd2(h2((hi & 0x000f000fu) | 0x64006400u), m1024), k3 = __hfma2(h2((hi & 0x00f000f0u) | 0x64006400u), sixteenth, m64);
            const uint4 y = make_uint4(u32(__hfma2(k0, s[0], z[0])), u32(__hfma2(k1, s[1], z[1])), u32(__hfma2(k2, s[2], z[2])), u32(__hfma2(k3, s[3], z[3])));
            *reinterpret_cast<uint4*>(op + (32 * i + e) * 128 + (((4 * half + t4) ^ ((d0 + e) & 7)) << 4)) = bad ? zero : y;
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&sh.v_full[vs]);
          mbar_arrive(&sh.raw_free[1][rs]);
        }
      }
    }
  } else {
    // ---------------- teams: a thread is a key, for half of the team's rows ----------------
    // After a wait that gave up the threads go on without waiting, through the same barriers.
    constexpr int kTeamThreads = 16 * kPgrSoft;
    const int sw = warp - 2, team = sw >> 3, side = (sw >> 2) & 1, qd = warp & 3, wt = (sw & 7) * 32 + lane, key = qd * 32 + lane, bar = 1 + team;
    const uint32_t lanes = static_cast<uint32_t>(qd * 32) << 16;
    const int width = team ? width1 : width0, c0 = side * (width / 16), c1 = c0 + width / 16;  // the thread's rows, in eights
    griddep_wait();
    griddep_launch();
    // Q: 16 lanes a row, 8 dims each, as vectors in the operand's order; a team its own rows, or half of the common ones
    {
      const int mine = two ? kPgrTeam : kPgrTeam / 2, from = two ? 0 : team * (kPgrTeam / 2), c8 = lane & 15;
      for (int i = (sw & 7) * 2 + (lane >> 4); i < mine; i += kPgrSoft) {
        const int qr = from + i, row = (two ? team * kPgrTeam : 0) + qr, q = row0 + row;
        uint4 in = make_uint4(0, 0, 0, 0);
        if (row < rows)
          in = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + (r.row + q / gq) * a.qs +
                                               static_cast<long long>(h * gq + q % gq) * kPgrD + c8 * 8);
        const uint32_t w[4] = {in.x, in.y, in.z, in.w};
        float y[8], big = 0.f, sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[2 * e] = __uint_as_float(w[e] << 16);
          y[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
          big = fmaxf(big, fmaxf(fabsf(y[2 * e]), fabsf(y[2 * e + 1])));
          sum += y[2 * e] + y[2 * e + 1];
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float up = query_scale(big), lo = up * 0.0625f;
        const uint4 v = make_uint4(pack_f16(y[0] * up, y[4] * up), pack_f16(y[1] * lo, y[5] * lo), pack_f16(y[2] * up, y[6] * up),
                                   pack_f16(y[3] * lo, y[7] * lo));
        *reinterpret_cast<uint4*>(sq + ((two ? team : 0) * 2 + (c8 >> 3)) * kPgrQ + qr * 128 + (((c8 & 7) ^ (qr & 7)) << 4)) = v;
        const float z1 = __shfl_down_sync(0xffffffffu, sum, 8);
        if (c8 == 0)
          for (int tt = two ? team : 0; tt <= (two ? team : 1); ++tt) {
            float* rc = reinterpret_cast<float*>(&sh.rc[tt][qr >> 1][0]) + (qr & 1);
            const bool live = row < rows;  // (others' weights are 0)
            rc[0] = live ? a.scale_log2 * 16777216.f / up : 0.f;
            rc[2] = live ? sum * a.scale_log2 : 0.f;
            rc[4] = live ? z1 * a.scale_log2 : 0.f;
            rc[6] = live ? FLT_MAX : -1000.f;
            sh.ref[tt][qr] = -FLT_MAX;  // (nothing seen)
          }
      }
    }
    fence_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.q_full);
    named_bar_sync(3, 32 * kPgrSoft);
    constexpr int kEights = kPgrTeam / 16;  // of a thread's rows
    f2_t l[4 * kEights];                    // the key's sums of p, by pairs of rows
#pragma unroll
    for (int i = 0; i < 4 * kEights; ++i) l[i] = f2_pack(0.f, 0.f);
    uint8_t* prow = sp + team * kPgrP + key * 128;
    const uint32_t s_at = tm + lanes + team * 128, o_at = tm + lanes + kPgrO + team * 64, rc_at = smem_u32(&sh.rc[team][0][0]);
    bool ok = true;
    int used = 0;
    for (int t = two ? 0 : team; t < n; t += two ? 1 : 2, ++used) {
      const int j = used, pb = t & 3;
      ok = ok && quiet_wait(&sh.par_full[pb], (t >> 2) & 1, abort, a.status) && quiet_wait(&sh.s_full[team], j & 1, abort, a.status) &&
           (j == 0 || quiet_wait(&sh.pv_done[team], (j - 1) & 1, abort, a.status));
      __syncwarp();
      tc_fence_after();
      const bool none = sh.bad[pb][qd >> 1] != 0;  // no such page
      const uint2 kp = sh.par[pb][key];
      const float vk = kp.x & 0x8000u ? 32.f : 1.f;  // what the key's weights are multiplied by for its values
      const float2 sz0 = __half22float2(h2(kp.x & 0xffff7fffu)), sz1 = __half22float2(h2(kp.y));
      const f2_t ks0 = f2_pack(sz0.x, sz0.x), kz0 = f2_pack(sz0.y, sz0.y), ks1 = f2_pack(sz1.x, sz1.x), kz1 = f2_pack(sz1.y, sz1.y);
      // every eight rows' exponents e - ref to use(eight, four pairs)
      const auto each = [&](int when, auto use) {
#pragma unroll
        for (int cc = 0; cc < kEights; ++cc) {
          const int c = c0 + cc;
          if (c >= c1) break;
          uint32_t s0[8], s1[8];
          tmem_ld8(s_at + c * 8, s0);
          tmem_ld8(s_at + 64 + c * 8, s1);
          tmem_here(s0, s1);
          f2_t e[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            f2_t f, ra, rb, nref;
            pairs_at(rc_at + (c * 4 + q) * 32, when, &f, &ra);
            pairs_at(rc_at + (c * 4 + q) * 32 + 16, when, &rb, &nref);
            const f2_t x0 = f2_pack(__uint_as_float(s0[2 * q]), __uint_as_float(s0[2 * q + 1]));
            const f2_t x1 = f2_pack(__uint_as_float(s1[2 * q]), __uint_as_float(s1[2 * q + 1]));
            const f2_t code = f2_fma(ks1, x1, f2_mul(ks0, x0));
            e[q] = f2_fma(code, f, f2_fma(kz0, ra, f2_fma(kz1, rb, nref)));
          }
          use(cc, e);
        }
      };
      // the tile's weights, into P and the sums; whether one passes kPgrTop
      const auto weights = [&](int when) {
        if (none) return false;
        __half2 top = __half2half2(__ushort_as_half(0));
        const f2_t vk2 = f2_pack(vk, vk);
        each(when, [&](int cc, const f2_t* e) {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 x = f2_unpack(e[i]);
            const f2_t y = f2_pack(ex2(x.x), ex2(x.y));
            l[cc * 4 + i] = f2_add(l[cc * 4 + i], y);
            const float2 v = f2_unpack(f2_mul(y, vk2));
            w[i] = pack_f16(v.x, v.y);
            top = __hmax2(top, h2(w[i]));
          }
          *reinterpret_cast<uint4*>(prow + (((c0 + cc) ^ (key & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
        });
        const float2 m = __half22float2(top);
        return fmaxf(m.x, m.y) > kPgrTop * vk;
      };
      if (none)
        for (int c = c0; c < c1; ++c) *reinterpret_cast<uint4*>(prow + ((c ^ (key & 7)) << 4)) = make_uint4(0, 0, 0, 0);
      const bool over = weights(2 * t);
      fence_async_smem();
      tc_fence_before();
      if (team_or(bar, over)) {
        // References rise.  The tile's sums are taken back (what an infinite weight leaves is scaled to nothing), the rows' maxima
        // over the keys found.
        tc_fence_after();
        if (!none) {
          each(2 * t, [&](int cc, const f2_t* e) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 x = f2_unpack(e[i]), was = f2_unpack(l[cc * 4 + i]);
              const float2 y = make_float2(ex2(x.x), ex2(x.y));
              l[cc * 4 + i] = f2_pack(y.x == INFINITY ? 0.f : was.x - y.x, y.y == INFINITY ? 0.f : was.y - y.y);
            }
          });
          // (scores without the references: the first tile's are the largest float)
#pragma unroll 1
          for (int c = c0; c < c1; ++c) {
            uint32_t s0[8], s1[8];
            tmem_ld8(s_at + c * 8, s0);
            tmem_ld8(s_at + 64 + c * 8, s1);
            tmem_here(s0, s1);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int q = c * 8 + i;
              const float* rc = reinterpret_cast<const float*>(&sh.rc[team][q >> 1][0]) + (q & 1);
              const float code = fmaf(sz1.x, __uint_as_float(s1[i]), sz0.x * __uint_as_float(s0[i]));
              float e = fmaf(code, rc[0], fmaf(sz0.y, rc[2], sz1.y * rc[4]));
#pragma unroll
              for (int o = 16; o > 0; o >>= 1) e = fmaxf(e, __shfl_xor_sync(0xffffffffu, e, o));
              if (lane == 0) sh.wmax[team][qd][q] = e;
            }
          }
        } else {
          for (int q = c0 * 8 + lane; q < c1 * 8; q += 32) sh.wmax[team][qd][q] = -INFINITY;
        }
        tc_fence_before();
        named_bar_sync(bar, kTeamThreads);
        if (wt < kPgrTeam) {
          const int row = (two ? team * kPgrTeam : 0) + wt;
          float fac = 1.f;
          if (row < rows) {
            const float most = fmaxf(fmaxf(sh.wmax[team][0][wt], sh.wmax[team][1][wt]), fmaxf(sh.wmax[team][2][wt], sh.wmax[team][3][wt]));
            const float ref = sh.ref[team][wt];
            if (most - ref > 9.f) {
              const float now = ceilf(most);
              fac = ref == -FLT_MAX ? 0.f : pow2(ref - now);
              sh.ref[team][wt] = now;
              (reinterpret_cast<float*>(&sh.rc[team][wt >> 1][1]) + (wt & 1))[2] = -now;
            }
          }
          sh.fac[team][wt] = fac;
        }
        named_bar_sync(bar, kTeamThreads);
        tc_fence_after();
#pragma unroll
        for (int i = 0; i < 4 * kEights; ++i)
          if (i < (c1 - c0) * 4) l[i] = f2_mul(l[i], *reinterpret_cast<const f2_t*>(&sh.fac[team][c0 * 8 + 2 * i]));
        if (j > 0)
#pragma unroll 1
          for (int c = c0; c < c1; ++c) {
            uint32_t o[8];
            tmem_ld8(o_at + c * 8, o);
            tmem_here(o);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * sh.fac[team][c * 8 + i]);
            tmem_st8(o_at + c * 8, o);
          }
        weights(2 * t + 1);
        fence_async_smem();
        tc_fence_before();
        named_bar_sync(bar, kTeamThreads);
      }
      if (wt == 0) mbar_arrive(&sh.p_full[team]);
    }
    // ---------------- the CTA's part: 128 dims by rows, references and sums ----------------
    ok = ok && (used == 0 || quiet_wait(&sh.pv_done[team], (used - 1) & 1, abort, a.status));
    __syncwarp();
    tc_fence_after();
#pragma unroll
    for (int i = 0; i < 4 * kEights; ++i) {
      float2 y = f2_unpack(l[i]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        y.x += __shfl_xor_sync(0xffffffffu, y.x, o);
        y.y += __shfl_xor_sync(0xffffffffu, y.y, o);
      }
      if (lane == 0 && i < (c1 - c0) * 4) *reinterpret_cast<float2*>(&sh.lsum[team][qd][c0 * 8 + 2 * i]) = y;
    }
    const int mine = two && !team ? kPgrTeam : rows - (two ? kPgrTeam : 0);  // the team's rows
    const long long slot = (static_cast<long long>(blockIdx.x) * 2 + team) * kPgrTeam;
    named_bar_sync(bar, kTeamThreads);
    if (wt < mine) {
      const float sum = (sh.lsum[team][0][wt] + sh.lsum[team][1][wt]) + (sh.lsum[team][2][wt] + sh.lsum[team][3][wt]);
      const float ref = sh.ref[team][wt];
      __stcg(p.part_ml + slot + wt, make_float2(ref == -FLT_MAX ? -INFINITY : ref, sum));
    }
    if (used > 0)
#pragma unroll 1
      for (int c = c0; c < c1; ++c) {
        uint32_t o[8];
        tmem_ld8(o_at + c * 8, o);
        tmem_here(o);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (c * 8 + i < mine) __stcg(p.part_o + (slot + c * 8 + i) * kPgrD + key, __uint_as_float(o[i]));
      }
    tc_fence_before();
    named_bar_sync(3, 32 * kPgrSoft);
    if (sw == 0 && lane == 0) {
      sh.last = atom_add_acq_rel_gpu(&p.counters[first_cta], 1) == splits - 1;
      if (sh.last) atomicExch(&p.counters[first_cta], 0);
    }
    named_bar_sync(3, 32 * kPgrSoft);
    if (sh.last) {
      // the item's last CTA: a warp joins a row's parts, every CTA's, or (up to 64 rows) both of its teams'
      const int parts = two ? splits : 2 * splits;
      for (int row = sw; row < rows; row += kPgrSoft) {
        const auto part = [&](int k) {
          const long long at = two ? (first_cta + k) * 2 + (row >> 6) : first_cta * 2 + k;
          return at * kPgrTeam + (row & (kPgrTeam - 1));
        };
        float M = -INFINITY, L = 0.f;
        for (int k = lane; k < parts; k += 32) M = fmaxf(M, __ldcg(p.part_ml + part(k)).x);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
        const float mb = M == -INFINITY ? 0.f : M;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k0 = 0; k0 < parts; k0 += 32) {
          const float2 ml = k0 + lane < parts ? __ldcg(p.part_ml + part(k0 + lane)) : make_float2(-INFINITY, 0.f);
          const float fw = ml.x == -INFINITY ? 0.f : ex2(ml.x - mb);
          L = fmaf(fw, ml.y, L);
          const int m = min(32, parts - k0);
          for (int k = 0; k < m; k += 4) {
            float4 y[4];
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              w[i] = __shfl_sync(0xffffffffu, fw, (k + i) & 31);
              // (a part that saw nothing has no outputs)
              const bool there = k + i < m && w[i] != 0.f;
              y[i] = there ? __ldcg(reinterpret_cast<const float4*>(p.part_o + part(k0 + k + i) * kPgrD) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              s.x = fmaf(w[i], y[i].x, s.x);
              s.y = fmaf(w[i], y[i].y, s.y);
              s.z = fmaf(w[i], y[i].z, s.z);
              s.w = fmaf(w[i], y[i].w, s.w);
            }
          }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
        finish_row<kPgrD>(p, r, h, row0 + row, lane, M, L, s);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tm, kPgrTmem);
  }
}

}  // namespace

cudaError_t paged_attn_group_prepare() {
  return cudaFuncSetAttribute(paged_attn_group_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kPgrSmem));
}

bool plan_paged_attention_group(PaShared& p, const PaTask* tasks, int n_tasks, int sms, int* grid) {
  if (!pa_plan(p, tasks, n_tasks, kPgrRows, kPgrKeys / 32)) return false;
  *grid = 0;
  if (p.n_req == 0) return true;
  // Runs within an item: the shortest that make a CTA an SM at most.
  const auto items = [&](int i) { return ((i + 1 < p.n_req ? p.r[i + 1].off : p.total) - p.r[i].off) / p.r[i].units; };
  const auto ctas = [&](int len) {
    long long c = 0;
    for (int i = 0; i < p.n_req; ++i) c += static_cast<long long>(items(i)) * ((p.r[i].units + len - 1) / len);
    return c;
  };
  int longest = 1;
  for (int i = 0; i < p.n_req; ++i) longest = p.r[i].units > longest ? p.r[i].units : longest;
  int len = 1;
  while (len < longest && ctas(len) > sms) ++len;
  if (ctas(len) > 2LL * sms) return false;  // (partial results have room for that)
  p.aligned = 1;
  int at = 0;
  for (int i = 0; i < p.n_req; ++i) {
    p.r[i].cta = at;
    p.r[i].splits = (p.r[i].units + len - 1) / len;
    at += items(i) * p.r[i].splits;
  }
  *grid = at;
  return true;
}

cudaError_t launch_paged_attention_group(const PaShared& p, int grid, cudaStream_t s) {
  return launch_k(paged_attn_group_kernel, dim3(grid), dim3(kPgrThreads), kPgrSmem, s, true, p);
}

}  // namespace tss
