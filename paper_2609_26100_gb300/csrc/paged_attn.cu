// Attention of draft blocks over the paged 4-bit cache.
//
// One CTA per (row, query head): its warps take every fourth visible key, a lane holds D / 32 dims of the
// query, keys and output, and each warp keeps the running maximum and sum of its softmax; the four parts
// are joined at the end.
#include "paged.h"

namespace tss {
namespace {

constexpr int kPaThreads = 128;

// Whether the row (position qp, ancestors anc) of request r sees key j.
__device__ __forceinline__ bool sees(const PgAttnParams& p, const PgReq& r, int i, int qp, const unsigned long long* anc, int j) {
  int kp = j;
  if (j >= r.first) {
    const int x = j - r.first;
    if (anc ? !(anc[x >> 6] >> (x & 63) & 1ull) : x > i) return false;
    if (p.window && p.positions) kp = max(p.positions[r.row + x], r.first);
  }
  return !p.window || qp - kp < p.window || j < p.sinks;
}

template <int D>
__global__ void __launch_bounds__(kPaThreads) paged_attn_kernel(const __grid_constant__ PgAttnParams p) {
  using B = PgBlock<D>;
  constexpr int N = D / 32;
  __shared__ float part[kPaThreads / 32][D + 2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = blockIdx.y, kvh = h / (p.hq / p.hk);
  const int row = blockIdx.x;
  int b = 0;
  while (b + 1 < p.batch.n_req && p.batch.r[b + 1].row <= row) ++b;
  while (p.batch.r[b].n == 0 && b > 0) --b;
  const PgReq r = p.batch.r[b];
  const int i = row - r.row;
  const int qp = p.window && p.positions ? max(p.positions[row], r.first) : r.first + i;
  const unsigned long long* anc = p.mask ? p.mask + 2LL * row : nullptr;
  float q[N], o[N] = {};
  const long long qo = row * p.qs + static_cast<long long>(h) * D + lane * N;
  if (p.is_half)
    load_vec<__half, N>(static_cast<const __half*>(p.q) + qo, q);
  else
    load_vec<__nv_bfloat16, N>(static_cast<const __nv_bfloat16*>(p.q) + qo, q);
  float m = -INFINITY, l = 0.f;
  const int lo = p.window ? max(0, r.first - p.window + 1) : 0;
  for (int j = warp; j < r.first + r.n; j += kPaThreads / 32) {
    if (j < lo && j >= p.sinks) continue;
    if (!sees(p, r, i, qp, anc, j)) continue;
    const int page = p.table[static_cast<long long>(r.seq) * p.max_pages + j / kPgTokens];
    if (page < 0 || page >= p.n_pages) {
      if (lane == 0) report(p.status, kStatusCheck);
      continue;
    }
    const uint8_t* blk = p.pool + (static_cast<long long>(page) * p.hk + kvh) * B::kBytes;
    const int t = j % kPgTokens, d0 = lane * N, g = d0 / kPgGroup;
    const uint8_t* kb = blk + B::kK + t * (D / 2) + (d0 % kPgGroup) / 16 * (D / 8) + g * 8 + (d0 % 16) / 2;
    const uint32_t kc = N == 4 ? *reinterpret_cast<const uint16_t*>(kb) : *kb;
    const float2 kp = __half22float2(reinterpret_cast<const __half2*>(blk + B::kKParams)[t * B::kGroups + g]);
    const float2 vp = __half22float2(reinterpret_cast<const __half2*>(blk + B::kVParams)[t * B::kGroups + g]);
    const uint32_t* vw = reinterpret_cast<const uint32_t*>(blk + B::kV) + (((t / 32) * (D / 4) + d0 / 4) * 4 + t % 8 / 2) * 4 + d0 % 4;
    const int shift = 4 * (t % 32 / 8 + 4 * (t & 1));
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) s = fmaf(q[e], fmaf(static_cast<float>(kc >> (4 * e) & 15u), kp.x, kp.y), s);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    s *= p.scale_log2;
    const float mn = fmaxf(m, s), a = exp2f(m - mn), w = exp2f(s - mn);
    l = l * a + w;
    m = mn;
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = o[e] * a + w * fmaf(static_cast<float>(vw[e] >> shift & 15u), vp.x, vp.y);
  }
#pragma unroll
  for (int e = 0; e < N; ++e) part[warp][lane * N + e] = o[e];
  if (lane == 0) {
    part[warp][D] = m;
    part[warp][D + 1] = l;
  }
  __syncthreads();
  if (warp > 0) return;
  float M = -INFINITY, L = 0.f;
  for (int w = 0; w < kPaThreads / 32; ++w) M = fmaxf(M, part[w][D]);
#pragma unroll
  for (int e = 0; e < N; ++e) o[e] = 0.f;
  for (int w = 0; w < kPaThreads / 32 && M > -INFINITY; ++w) {
    const float f = exp2f(part[w][D] - M);
    L += f * part[w][D + 1];
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] += f * part[w][lane * N + e];
  }
#pragma unroll
  for (int e = 0; e < N; ++e) o[e] = L > 0.f ? o[e] / L : L == 0.f ? 0.f : L;  // (a NaN stays one)
  const long long oo = row * p.os + static_cast<long long>(h) * D + lane * N;
  if (p.is_half)
    store_vec<__half, N>(static_cast<__half*>(p.out) + oo, o);
  else
    store_vec<__nv_bfloat16, N>(static_cast<__nv_bfloat16*>(p.out) + oo, o);
  if (lane == 0 && p.lse) p.lse[static_cast<long long>(row) * p.hq + h] = (M + log2f(L)) * 0.6931471805599453f;
}

}  // namespace

cudaError_t launch_paged_attention(const tss_paged* h, const PgAttnParams& p, int rows, cudaStream_t s) {
  const dim3 grid(rows, h->hq);
  if (h->d == 64)
    paged_attn_kernel<64><<<grid, kPaThreads, 0, s>>>(p);
  else
    paged_attn_kernel<128><<<grid, kPaThreads, 0, s>>>(p);
  return cudaGetLastError();
}

}  // namespace tss
