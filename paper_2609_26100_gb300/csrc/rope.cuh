// Per-head norms and the rotary rotation of rows, as rope.cu and append_rope.cu do them: the same operations in the same
// order, so that a head gets the same bits in both.
#pragma once

#include "ops.cuh"

namespace tss {

struct RopeParams {
  int rows, hq, hk, d, rot, max_pos;
  int splits;  // warps that share a row's head groups
  const void *q, *k;
  void *q_out, *k_out;
  long long qs, ks, qos, kos;
  const void *q_gain, *k_gain;
  float eps;
  const float* table;
  const int* positions;
  int* status;
};

constexpr int kRopeThreads = 128;

// A lane's 16 elements of a head as two vectors of 8, from elements c0 and c1, that contain both members of its pairs.
template <int LANES, bool INTER>
struct RopeLane {
  int j, c0, c1;
  bool live, turns;
  __device__ __forceinline__ RopeLane(const RopeParams& p, int lane) {
    j = lane & (LANES - 1);
    live = 16 * j < p.d;
    turns = 16 * j < p.rot;
    const int rs = p.rot >> 4;
    c0 = INTER || !turns ? 16 * j : 8 * j;
    c1 = INTER || !turns ? 16 * j + 8 : 8 * (j + rs);
  }
};

// The row's position, kept within the table.
__device__ __forceinline__ int rope_position(const RopeParams& p, long long row) {
  const int pos = p.positions[row];
  if (pos >= 0 && pos < p.max_pos) return pos;
  report(p.status, kStatusCheck);
  return pos < 0 ? 0 : p.max_pos - 1;
}

// 1 / sqrt(mean(x^2) + eps) of a head whose sum of squares is ss, and x r gain of the lane's elements.
__device__ __forceinline__ float rope_scale(float ss, const RopeParams& p) { return 1.f / sqrtf(ss / static_cast<float>(p.d) + p.eps); }
__device__ __forceinline__ void rope_norm(float* a, const float* g, float r) {
#pragma unroll
  for (int i = 0; i < 16; ++i) a[i] = a[i] * r * g[i];
}

// The rotation of the lane's eight pairs by their (cos, sin); the second products are rounded, the first are not.
template <bool INTER>
__device__ __forceinline__ void rope_turn(float* a, const float* cs) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float& u = INTER ? a[2 * i] : a[i];
    float& v = INTER ? a[2 * i + 1] : a[8 + i];
    const float c = cs[2 * i], s = cs[2 * i + 1], u0 = u, v0 = v;
    u = fmaf(u0, c, -__fmul_rn(v0, s));
    v = fmaf(u0, s, __fmul_rn(v0, c));
  }
}

// The head groups of a row that warp w has.  LANES: lanes of one head (a power of two, at least d / 16).
template <typename T, int LANES, bool INTER>
__device__ __forceinline__ void rope_row(const RopeParams& p, long long w, int lane) {
  constexpr int kHeads = 32 / LANES;  // heads of a group: one turn of a warp
  const long long row = w / p.splits;
  const int part = static_cast<int>(w - row * p.splits);
  if (row >= p.rows) return;
  const RopeLane<LANES, INTER> at(p, lane);
  const int sub = lane / LANES, c0 = at.c0, c1 = at.c1;
  const bool live = at.live, turns = at.turns;
  float cs[16];
  if (turns) load_vec<float, 16>(p.table + static_cast<size_t>(rope_position(p, row)) * p.rot + 16 * at.j, cs);
  const int heads = p.hq + p.hk, step = p.splits * kHeads;
  // the next head's vectors are on their way while this one is worked on
  Raw8<T> next[2];
  const auto fetch = [&](int h) {
    if (live && h < heads) {
      const T* x = h < p.hq ? static_cast<const T*>(p.q) + row * p.qs + static_cast<long long>(h) * p.d
                            : static_cast<const T*>(p.k) + row * p.ks + static_cast<long long>(h - p.hq) * p.d;
      next[0].load(x + c0);
      next[1].load(x + c1);
    }
  };
  fetch(part * kHeads + sub);
#pragma unroll 1
  for (int h = part * kHeads + sub; h - sub < heads; h += step) {
    const bool on = live && h < heads, isq = h < p.hq;
    T* y = isq ? static_cast<T*>(p.q_out) + row * p.qos + static_cast<long long>(h) * p.d
               : static_cast<T*>(p.k_out) + row * p.kos + static_cast<long long>(h - p.hq) * p.d;
    const T* gain = static_cast<const T*>(isq ? p.q_gain : p.k_gain);
    float a[16];
    next[0].to(a);
    next[1].to(a + 8);
    fetch(h + step);
    // (every lane of the warp takes part in the butterfly; the condition is the same for all)
    if (p.q_gain || p.k_gain) {
      float ss = 0.f;
      if (on) {
#pragma unroll
        for (int i = 0; i < 16; ++i) ss = fmaf(a[i], a[i], ss);
      }
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (on && gain) {
        const float r = rope_scale(ss, p);
        float g[16];
        load_vec<T, 8>(gain + c0, g);
        load_vec<T, 8>(gain + c1, g + 8);
        rope_norm(a, g, r);
      }
    }
    if (!on) continue;
    if (turns) rope_turn<INTER>(a, cs);
    store_vec<T, 8>(y + c0, a);
    store_vec<T, 8>(y + c1, a + 8);
  }
}

// Warps of a row of `heads` heads: a warp per (row, head group) until there are as many warps as the GPU holds; then fewer
// warps per row, each with more groups, so that the table row is read less often.
inline int rope_splits(int rows, int heads, int lanes) {
  const long long want = 152LL * 64;
  int splits = (heads + 32 / lanes - 1) / (32 / lanes);
  while (splits > 1 && static_cast<long long>(rows) * ((splits + 1) / 2) >= want) splits = (splits + 1) / 2;
  return splits;
}

// Checks the arguments of a call (those of tss_qk_rope; `to_pages`: of one that may leave k_out out) and lays them out; *lanes:
// of a head.  p->rows is 0 where there is nothing to do.
tss_status take_rope(const tss_rope_args* a, bool to_pages, RopeParams* p, int* lanes);

}  // namespace tss
