// Per-head norms of queries and keys with the rotary position rotation, in one pass over the rows.
//
//   x' = x rsqrt(mean(x^2) + eps) gain;  (a, b) -> (a cos - b sin, b cos + a sin)
//
// A lane holds 16 elements of a head as two vectors of 8 that contain both members of its pairs: in the
// half layout vectors j and j + rot/16, in the interleaved one 2j and 2j + 1.  Either way its pairs are
// 8 consecutive ones, 8j .. 8j + 7, so one 64-byte read of the table serves the lane for every head of
// the row.  The mean of squares is a butterfly over the head's lanes (8 at head_dim 128, four heads to a
// warp).
//
// Bound: HBM, each element read and written once: 4096 rows of 64 heads of 128, bf16, with norms 26 us, 5.1 TB/s.  A step of
// 6 rows 2.3 us: launch and two dependent loads (position, table).  The next head's vectors are held as they come: widened
// to fp32 while in flight they cost registers and 38 us.
#include "rope.cuh"

namespace tss {
namespace {

template <typename T, int LANES, bool INTER>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeParams p) {
  griddep_wait();
  griddep_launch();
  rope_row<T, LANES, INTER>(p, static_cast<long long>(blockIdx.x) * (kRopeThreads / 32) + (threadIdx.x >> 5), threadIdx.x & 31);
}

struct RopeFreq {
  double f[128];
};

// One thread per (position, pair): the angle in double, so that it is right to the last bits of fp32 at
// any position.
__global__ void __launch_bounds__(256) rope_table_kernel(const __grid_constant__ RopeFreq freq, int n_pairs, double factor,
                                                         long long n, float2* table) {
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) {
    const long long pos = i / n_pairs;
    double s, c;
    sincos(static_cast<double>(pos) * freq.f[i - pos * n_pairs], &s, &c);
    table[i] = make_float2(static_cast<float>(c * factor), static_cast<float>(s * factor));
  }
}

template <typename T, int LANES>
cudaError_t rope_launch(const RopeParams& p, bool inter, unsigned grid, cudaStream_t s) {
  return launch_k(inter ? rope_kernel<T, LANES, true> : rope_kernel<T, LANES, false>, dim3(grid), dim3(kRopeThreads), 0, s, true, p);
}

template <typename T>
cudaError_t rope_dispatch(const RopeParams& p, bool inter, unsigned grid, cudaStream_t s, int lanes) {
  switch (lanes) {
    case 1: return rope_launch<T, 1>(p, inter, grid, s);
    case 2: return rope_launch<T, 2>(p, inter, grid, s);
    case 4: return rope_launch<T, 4>(p, inter, grid, s);
    case 8: return rope_launch<T, 8>(p, inter, grid, s);
    default: return rope_launch<T, 16>(p, inter, grid, s);
  }
}

}  // namespace

tss_status take_rope(const tss_rope_args* a, bool to_pages, RopeParams* p, int* lanes) {
  *p = RopeParams{};
  if (!a) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  if (a->n_rows < 0 || a->n_q_heads < 0 || a->n_k_heads < 0 || a->n_q_heads > (1 << 16) || a->n_k_heads > (1 << 16))
    return refuse(TSS_ERR_INVALID_ARG, "n_rows must be >= 0 and the head counts in [0, 65536]");
  if (a->head_dim < 16 || a->head_dim > 256 || a->head_dim % 16)
    return refuse(TSS_ERR_INVALID_ARG, "head_dim must be a multiple of 16 in [16, 256]");
  if (a->rot_dim < 0 || a->rot_dim > a->head_dim || a->rot_dim % 16)
    return refuse(TSS_ERR_INVALID_ARG, "rot_dim must be a multiple of 16 in [0, head_dim]");
  if (!known_dtype(a->dtype)) return refuse(TSS_ERR_INVALID_ARG, "unknown dtype");
  if (a->n_rows == 0 || a->n_q_heads + a->n_k_heads == 0) return TSS_OK;
  const struct {
    const void *in, *gain;
    void* out;
    int64_t is, os;
    int heads;
  } sides[2] = {{a->q, a->q_gain, a->q_out, a->q_stride, a->q_out_stride, a->n_q_heads},
                {a->k, a->k_gain, a->k_out, a->k_stride, a->k_out_stride, a->n_k_heads}};
  for (const auto& x : sides) {
    if (x.heads == 0) continue;
    const int64_t width = static_cast<int64_t>(x.heads) * a->head_dim;
    const bool out = !(to_pages && &x == &sides[1] && !x.out);
    if (!x.in || (out && !x.out)) return refuse(TSS_ERR_INVALID_ARG, "q and k need an input and an output");
    if (!aligned16(x.in) || !aligned16(x.out) || (x.gain && !aligned16(x.gain)))
      return refuse(TSS_ERR_INVALID_ARG, "q, k, their outputs and gains must be 16-byte aligned");
    if (!good_stride(x.is, width, a->dtype) || (out && !good_stride(x.os, width, a->dtype)))
      return refuse(TSS_ERR_INVALID_ARG, "row strides must hold the heads and be multiples of 16 bytes");
    if (x.in == x.out && x.is != x.os) return refuse(TSS_ERR_INVALID_ARG, "in place the strides must be equal");
  }
  if (a->rot_dim > 0) {
    if (!a->table || !a->positions) return refuse(TSS_ERR_INVALID_ARG, "rotation needs a table and positions");
    if (!aligned16(a->table)) return refuse(TSS_ERR_INVALID_ARG, "the table must be 16-byte aligned");
    if (a->max_positions < 1) return refuse(TSS_ERR_INVALID_ARG, "max_positions must be >= 1");
  }
  if ((a->q_gain || a->k_gain) && !(a->eps >= 0.f)) return refuse(TSS_ERR_INVALID_ARG, "eps must be >= 0");
  p->rows = a->n_rows;
  p->hq = a->n_q_heads;
  p->hk = a->n_k_heads;
  p->d = a->head_dim;
  p->rot = a->rot_dim;
  p->max_pos = a->max_positions;
  p->q = a->q;
  p->k = a->k;
  p->q_out = a->q_out;
  p->k_out = a->k_out;
  p->qs = a->q_stride;
  p->ks = a->k_stride;
  p->qos = a->q_out_stride;
  p->kos = a->k_out_stride;
  p->q_gain = a->n_q_heads ? a->q_gain : nullptr;
  p->k_gain = a->n_k_heads ? a->k_gain : nullptr;
  p->eps = a->eps;
  p->table = a->table;
  p->positions = a->positions;
  p->status = a->status;
  *lanes = 1;
  while (*lanes * 16 < p->d) *lanes *= 2;
  return TSS_OK;
}

}  // namespace tss

using namespace tss;

extern "C" tss_status tss_qk_rope(const tss_rope_args* a, void* stream) {
  RopeParams p;
  int lanes = 1;
  const tss_status st = take_rope(a, false, &p, &lanes);
  if (st != TSS_OK || p.rows == 0) return st;
  p.splits = rope_splits(p.rows, p.hq + p.hk, lanes);
  const long long warps = static_cast<long long>(p.rows) * p.splits, per = kRopeThreads / 32;
  if ((warps + per - 1) / per > 0x7fffffffLL) return refuse(TSS_ERR_INVALID_ARG, "too many rows for one launch");
  const unsigned grid = static_cast<unsigned>((warps + per - 1) / per);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool inter = a->interleaved != 0;
  const cudaError_t e = a->dtype == TSS_DTYPE_BF16  ? rope_dispatch<__nv_bfloat16>(p, inter, grid, s, lanes)
                        : a->dtype == TSS_DTYPE_F16 ? rope_dispatch<__half>(p, inter, grid, s, lanes)
                                                    : rope_dispatch<float>(p, inter, grid, s, lanes);
  return e == cudaSuccess ? TSS_OK : refuse_cuda(e, "launch");
}

extern "C" tss_status tss_rope_frequencies(int kind, int rot_dim, double theta, double factor, double original,
                                           double* inv_freq, double* attention_factor) {
  if (!inv_freq || !attention_factor) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  if (rot_dim < 2 || rot_dim % 2) return refuse(TSS_ERR_INVALID_ARG, "rot_dim must be even and positive");
  if (!(theta > 1.0) || !(theta < 1e300)) return refuse(TSS_ERR_INVALID_ARG, "theta must be above 1 and finite");
  if (kind < TSS_ROPE_NONE || kind > TSS_ROPE_BANDS) return refuse(TSS_ERR_INVALID_ARG, "unknown kind of scaling");
  if (kind != TSS_ROPE_NONE && (!(factor >= 1.0) || !(factor < 1e9)))
    return refuse(TSS_ERR_INVALID_ARG, "factor must be in [1, 1e9)");
  if ((kind == TSS_ROPE_YARN || kind == TSS_ROPE_BANDS) && (!(original >= 1.0) || !(original < 1e12)))
    return refuse(TSS_ERR_INVALID_ARG, "original must be in [1, 1e12)");
  if (kind == TSS_ROPE_NTK && rot_dim < 4) return refuse(TSS_ERR_INVALID_ARG, "NTK scaling needs rot_dim >= 4");
  const double turn = 6.283185307179586476925286766559;
  const int n = rot_dim / 2;
  *attention_factor = 1.0;
  const double base = kind == TSS_ROPE_NTK ? theta * pow(factor, static_cast<double>(rot_dim) / (rot_dim - 2)) : theta;
  // YARN: the (fractional) pair index whose frequency turns `t` times within the original context
  double lo = 0, hi = 0;
  if (kind == TSS_ROPE_YARN) {
    const auto index = [&](double t) { return rot_dim * log(original / (turn * t)) / (2 * log(theta)); };
    lo = fmax(0.0, floor(index(32.0)));
    // (past the last pair, n - 1, where even that one turns more than once: it is not divided by all of the factor then)
    hi = fmin(static_cast<double>(rot_dim - 1), ceil(index(1.0)));
    if (hi - lo < 1e-3) hi = lo + 1e-3;
    *attention_factor = 0.1 * log(factor) + 1.0;
  }
  for (int i = 0; i < n; ++i) {
    double f = pow(base, -2.0 * i / rot_dim);
    if (kind == TSS_ROPE_LINEAR) f /= factor;
    if (kind == TSS_ROPE_YARN) {
      const double ramp = fmin(1.0, fmax(0.0, (i - lo) / (hi - lo)));
      f = f * (1.0 - ramp) + f / factor * ramp;
    }
    if (kind == TSS_ROPE_BANDS) {
      const double wave = turn / f;
      if (wave > original) {
        f /= factor;
      } else if (wave > original / 4) {
        const double keep = (original / wave - 1.0) / 3.0;  // 1 at original / 4, 0 at original
        f = f * keep + f / factor * (1.0 - keep);
      }
    }
    inv_freq[i] = f;
  }
  return TSS_OK;
}

extern "C" tss_status tss_rope_table(const double* inv_freq, int n_pairs, double attention_factor, int max_positions,
                                     float* table, void* stream) {
  if (!inv_freq || !table) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  if (n_pairs < 1 || n_pairs > 128) return refuse(TSS_ERR_INVALID_ARG, "n_pairs must be in [1, 128]");
  if (max_positions < 1) return refuse(TSS_ERR_INVALID_ARG, "max_positions must be >= 1");
  if (reinterpret_cast<uintptr_t>(table) & 7u) return refuse(TSS_ERR_INVALID_ARG, "the table must be 8-byte aligned");
  RopeFreq f{};
  for (int i = 0; i < n_pairs; ++i) f.f[i] = inv_freq[i];
  const long long n = static_cast<long long>(max_positions) * n_pairs;
  const unsigned grid = static_cast<unsigned>(n + 255 < 152LL * 8 * 256 ? (n + 255) / 256 : 152 * 8);
  rope_table_kernel<<<grid, 256, 0, static_cast<cudaStream_t>(stream)>>>(f, n_pairs, attention_factor, n,
                                                                          reinterpret_cast<float2*>(table));
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? TSS_OK : refuse_cuda(e, "launch");
}
