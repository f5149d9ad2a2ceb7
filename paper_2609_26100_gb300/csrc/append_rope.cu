// Appending keys and values to the paged 4-bit cache with the norms and the rotation on the way: tss_qk_rope and
// tss_paged_append in one launch.
//
//   q' = T(rot(norm(q))),  k' = T(rot(norm(k))),  pages <- quantised k', v       (T: the input's type)
//
// k' is rounded to T before it is quantised, so that the pages do not depend on the way that was taken: both use the same
// code (rope.cuh, paged_quant.cuh).  Half a step of T is 2^-9 of a value (bf16), of a code 2^-5 of the group's range.
//
// Warps that quantise K take a (request, 32-token half page, KV head) as in paged_quant.cuh: a lane rotates 16 elements of a
// token, which lie where its pairs do, and leaves them in shared memory, from where the warp picks up 8 neighbouring dims a
// lane to quantise.  Warps of V read the caller's rows, those after them rotate the rows' query heads.
//
// Bound: of few rows the launch and three dependent loads (position or page, table row, rows): 16 rows of 32 heads 5.7 us cold, where the
// two calls are two launches.  Of many rows issue slots and latency, with 20 warps an SM: 7171 rows of 32 heads, bf16, 89 us (3.0
// TB/s; the two calls 94), 68 of them for K and V (46 where neither is rotated by the call).
// Slower for the same rows: K's partners by shuffles in the lanes that quantise, without shared memory (156 us: 4 shuffles a vector and
// norms taken twice), the next table row or two turns' rows in flight (registers: 103, 109).
#include "paged_quant.cuh"
#include "rope.cuh"

namespace tss {
namespace {

struct ArParams {
  PqParams p;
  RopeParams r;       // of k; its q side is the query heads'
  long long quant;    // warps that quantise
};

// Rotated heads of a run's tokens to tile [tokens][D], and to k_out where there is one.
template <typename T, int D, bool INTER>
__device__ __forceinline__ void rope_run(const RopeParams& r, const PqUnit& u, T* tile, int lane) {
  constexpr int LANES = D / 16, kTok = 32 / LANES;
  const RopeLane<LANES, INTER> at(r, lane);
  const int sub = lane / LANES, n = u.hi - u.lo;
  int my_pos = 0;
  if (r.rot > 0 && lane < n) my_pos = rope_position(r, u.row + lane);
  Raw8<T> gain[2];
  if (r.k_gain) {
    gain[0].load(static_cast<const T*>(r.k_gain) + at.c0);
    gain[1].load(static_cast<const T*>(r.k_gain) + at.c1);
  }
  const T* src = static_cast<const T*>(r.k) + u.row * r.ks + static_cast<long long>(u.head) * D;
  T* out = r.k_out ? static_cast<T*>(r.k_out) + u.row * r.kos + static_cast<long long>(u.head) * D : nullptr;
  Raw8<T> next[2];
  const auto fetch = [&](int tok) {
    if (tok < n) {
      next[0].load(src + tok * r.ks + at.c0);
      next[1].load(src + tok * r.ks + at.c1);
    }
  };
  fetch(sub);
#pragma unroll 1
  for (int t0 = 0; t0 < n; t0 += kTok) {
    const int tok = t0 + sub;
    const bool on = tok < n;
    const int pos = __shfl_sync(0xffffffffu, my_pos, tok & 31);
    float cs[16], a[16];
    if (on && at.turns) load_vec<float, 16>(r.table + static_cast<size_t>(pos) * r.rot + 16 * at.j, cs);
    next[0].to(a);
    next[1].to(a + 8);
    fetch(tok + kTok);
    if (r.k_gain) {
      float ss = 0.f;
      if (on) {
#pragma unroll
        for (int i = 0; i < 16; ++i) ss = fmaf(a[i], a[i], ss);
      }
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      const float scale = rope_scale(ss, r);
      float g[16];
      gain[0].to(g);
      gain[1].to(g + 8);
      rope_norm(a, g, scale);
    }
    if (!on) continue;
    if (at.turns) rope_turn<INTER>(a, cs);
    store_vec<T, 8>(tile + tok * D + at.c0, a);
    store_vec<T, 8>(tile + tok * D + at.c1, a + 8);
    if (out) {
      store_vec<T, 8>(out + tok * r.kos + at.c0, a);
      store_vec<T, 8>(out + tok * r.kos + at.c1, a + 8);
    }
  }
  __syncwarp();
}

// Heads of 128 that turn as a whole, in the half layout: a lane's two vectors of a token are of one group of 64 dims each, 8 lanes a
// token, as the codes want them (scale_of: of two tokens at a time, both groups), so that nothing goes through shared memory (K and V of 7171 rows
// of 32 heads 68 us, 72 through it).
template <typename T>
__device__ __forceinline__ void rope_and_quantise(const PqParams& p, const RopeParams& r, PqUnit& u, int lane) {
  constexpr int D = 128;
  using B = PgBlock<D>;
  const RopeLane<8, false> at(r, lane);
  const int sub = lane >> 3, n = u.hi - u.lo;
  const T* src = static_cast<const T*>(r.k) + u.row * r.ks + static_cast<long long>(u.head) * D;
  T* out = r.k_out ? static_cast<T*>(r.k_out) + u.row * r.kos + static_cast<long long>(u.head) * D : nullptr;
  Raw8<T> next[2][2], gain[2];
  const auto fetch = [&](int i, int tok) {
    if (tok < n) {
      next[i][0].load(src + tok * r.ks + at.c0);
      next[i][1].load(src + tok * r.ks + at.c1);
    }
  };
  fetch(0, sub);
  fetch(1, sub + 4);
  const int my_pos = lane < n ? rope_position(r, u.row + lane) : 0;
  if (r.k_gain) {
    gain[0].load(static_cast<const T*>(r.k_gain) + at.c0);
    gain[1].load(static_cast<const T*>(r.k_gain) + at.c1);
  }
  pq_resolve(p, B::kBytes, lane, &u);
  if (!u.block && !out) return;
  const int tok0 = u.tok0 + u.lo;
  __half2* params = reinterpret_cast<__half2*>(u.block + B::kKParams) + tok0 * B::kGroups;
  uint8_t* krow = u.block + B::kK + tok0 * (D / 2) + PqLane<D>(at.j).k_at;
#pragma unroll 1
  for (int t0 = 0; t0 < n; t0 += 8) {
    Raw8<T> now[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int tok = t0 + 4 * i + sub;
      const bool on = tok < n;
      const int pos = __shfl_sync(0xffffffffu, my_pos, tok & 31);
      float cs[16], x[16];
      if (on) load_vec<float, 16>(r.table + static_cast<size_t>(pos) * D + 16 * at.j, cs);
      next[i][0].to(x);
      next[i][1].to(x + 8);
      fetch(i, tok + 8);
      if (r.k_gain) {
        float ss = 0.f;
        if (on) {
#pragma unroll
          for (int e = 0; e < 16; ++e) ss = fmaf(x[e], x[e], ss);
        }
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float scale = rope_scale(ss, r);
        float g[16];
        gain[0].to(g);
        gain[1].to(g + 8);
        rope_norm(x, g, scale);
      }
      now[2 * i].clear();
      now[2 * i + 1].clear();
      if (!on) continue;
      rope_turn<false>(x, cs);
      store_vec<T, 8>(reinterpret_cast<T*>(now[2 * i].v), x);
      store_vec<T, 8>(reinterpret_cast<T*>(now[2 * i + 1].v), x + 8);
      if (out) {
        *reinterpret_cast<uint4*>(out + tok * r.kos + at.c0) = now[2 * i].v[0];
        *reinterpret_cast<uint4*>(out + tok * r.kos + at.c1) = now[2 * i + 1].v[0];
      }
    }
    if (!u.block) continue;
    bool inside;
    const __half2 scales = scale_of(now, lane, &inside);
    inside = __all_sync(0xffffffffu, inside);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int tok = t0 + 4 * (k >> 1) + sub;
      const __half2 sz = __shfl_sync(0xffffffffu, scales, (lane & 24) | k);
      const uint32_t w = codes_of(now[k], sz, inside);
      if (tok >= n) continue;
      if (at.j == 0) params[tok * B::kGroups + (k & 1)] = sz;
      *reinterpret_cast<uint32_t*>(krow + tok * (D / 2) + (k & 1) * 8) = w;
    }
  }
}

// WHOLE: K by rope_and_quantise.  (Of 16-bit rows five CTAs an SM: 7171 rows of 32 heads through shared memory 93 us, with six 97, with
// seven 107: registers spill.)
template <typename T, int D, bool INTER, bool WHOLE>
__global__ void __launch_bounds__(kPqThreads, sizeof(T) == 4 ? 4 : 5) append_rope_kernel(const __grid_constant__ ArParams a) {
  extern __shared__ __align__(16) uint8_t ar_dyn[];
  const int lane = threadIdx.x & 31;
  griddep_wait();
  griddep_launch();
  const long long w = pq_warp();
  if (w >= a.quant) {
    // (without query heads the last CTA's spare warps come here, and a row has no splits)
    if (a.r.hq > 0) rope_row<T, D / 16, INTER>(a.r, w - a.quant, lane);
    return;
  }
  PqUnit u;
  if (!pq_unit(a.p, w, lane, &u)) return;
  if (u.side) {
    quantise_run<T, D>(a.p, u, static_cast<const T*>(a.p.v) + u.row * a.p.vs + u.head * D, a.p.vs, lane);
  } else if constexpr (WHOLE) {
    rope_and_quantise<T>(a.p, a.r, u, lane);
  } else {
    T* tile = reinterpret_cast<T*>(ar_dyn) + (threadIdx.x >> 5) * (32 * D);
    rope_run<T, D, INTER>(a.r, u, tile, lane);
    quantise_run<T, D>(a.p, u, tile, static_cast<long long>(D), lane);
  }
}

constexpr int ar_smem(int bytes, int d) { return kPqThreads / 32 * 32 * d * bytes; }

template <typename T, int D>
cudaError_t ar_launch(const ArParams& a, bool inter, unsigned grid, cudaStream_t s) {
  if constexpr (sizeof(T) == 2 && D == 128)
    if (!inter && a.r.rot == D) return launch_k(append_rope_kernel<T, D, false, true>, dim3(grid), dim3(kPqThreads), 0, s, true, a);
  return launch_k(inter ? append_rope_kernel<T, D, true, false> : append_rope_kernel<T, D, false, false>, dim3(grid), dim3(kPqThreads),
                  ar_smem(sizeof(T), D), s, true, a);
}
template <typename T>
cudaError_t ar_dispatch(const ArParams& a, bool inter, int d, unsigned grid, cudaStream_t s) {
  return d == 64 ? ar_launch<T, 64>(a, inter, grid, s) : ar_launch<T, 128>(a, inter, grid, s);
}

}  // namespace

// (of fp32 rows of 128 dims the tiles pass the 48 KiB that need no asking)
cudaError_t append_rope_prepare() {
  const int bytes = ar_smem(4, 128);
  const cudaError_t e = cudaFuncSetAttribute(append_rope_kernel<float, 128, false, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  return e == cudaSuccess ? cudaFuncSetAttribute(append_rope_kernel<float, 128, true, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) : e;
}

}  // namespace tss

using namespace tss;

extern "C" tss_status tss_paged_append_rope(tss_paged* h, const tss_paged_cache* cache, int layer, const tss_paged_batch* batch,
                                            const tss_rope_args* rope, const void* v, int64_t v_stride, void* stream) {
  ArParams a{};
  long long rows = 0;
  tss_status st = pq_take(h, cache, layer, batch, &a.p, &rows);
  int lanes = 1;
  if (st == TSS_OK) st = take_rope(rope, true, &a.r, &lanes);
  if (st != TSS_OK) return st;
  if (!pq_once(a.p.batch)) return refuse(TSS_ERR_INVALID_ARG, "a sequence appears twice");
  if (rope->n_k_heads != h->hk || rope->head_dim != h->d) return refuse(TSS_ERR_INVALID_ARG, "n_k_heads and head_dim must be the cache's");
  if (rope->n_rows != rows) return refuse(TSS_ERR_INVALID_ARG, "n_rows must be the batch's rows");
  if (rows == 0) return TSS_OK;
  if (!v || !aligned16(v) || !good_stride(v_stride, static_cast<int64_t>(h->hk) * h->d, rope->dtype))
    return refuse(TSS_ERR_INVALID_ARG, "v must be 16-byte aligned, its row stride hold the heads and be a multiple of 16 bytes");
  a.p.v = v;
  a.p.vs = v_stride;
  if (!a.r.status) a.r.status = h->status;
  a.quant = static_cast<long long>(a.p.total) * 2 * h->hk;
  a.r.hk = 0;  // (the warps of rows have the query heads alone)
  a.r.splits = rope_splits(a.r.rows, a.r.hq, lanes);
  const long long warps = a.quant + (a.r.hq ? static_cast<long long>(a.r.rows) * a.r.splits : 0), per = kPqThreads / 32;
  if ((warps + per - 1) / per > 0x7fffffffLL) return refuse(TSS_ERR_INVALID_ARG, "too many rows for one launch");
  const unsigned grid = static_cast<unsigned>((warps + per - 1) / per);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool inter = rope->interleaved != 0;
  const cudaError_t e = rope->dtype == TSS_DTYPE_BF16  ? ar_dispatch<__nv_bfloat16>(a, inter, h->d, grid, s)
                        : rope->dtype == TSS_DTYPE_F16 ? ar_dispatch<__half>(a, inter, h->d, grid, s)
                                                       : ar_dispatch<float>(a, inter, h->d, grid, s);
  return e == cudaSuccess ? TSS_OK : refuse_cuda(e, "launch");
}
