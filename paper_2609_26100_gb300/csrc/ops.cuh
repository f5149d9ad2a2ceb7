// What the stand-alone operators (rope.cu, paged.cu, paged_attn.cu, pages.cu) share: element types,
// vectors of eight elements, the layout of a 4-bit page, host-side refusals.
#pragma once

#include <new>
#include <string>

#include "internal.h"

namespace tss {

// ------------------------------------------------------------------------------------------
// Host
// ------------------------------------------------------------------------------------------
inline tss_status refuse(tss_status s, const char* msg) noexcept {
  try {
    set_last_error(msg);
  } catch (...) {  // no memory for the message: the status stands
  }
  return s;
}
inline tss_status refuse_cuda(cudaError_t e, const char* what) noexcept {
  cudaGetLastError();  // (a launch error is not sticky; leave none for the next call)
  try {
    set_last_error(std::string(what) + ": " + cudaGetErrorString(e));
  } catch (...) {
  }
  return TSS_ERR_CUDA;
}
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int dtype_bytes(int dtype) { return dtype == TSS_DTYPE_F32 ? 4 : 2; }
inline bool known_dtype(int dtype) { return dtype == TSS_DTYPE_BF16 || dtype == TSS_DTYPE_F16 || dtype == TSS_DTYPE_F32; }
// A row stride (elements) of rows of `width` elements that keeps them apart and 16-byte aligned.
inline bool good_stride(int64_t stride, int64_t width, int dtype) {
  return stride >= width && stride < (int64_t(1) << 40) && (stride * dtype_bytes(dtype)) % 16 == 0;
}
// The current device and its SM count, if it is an sm_103.
inline tss_status this_device(int* dev, int* sms) {
  int major = 0, minor = 0;
  cudaError_t e = cudaGetDevice(dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, *dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, *dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *dev);
  if (e != cudaSuccess) return refuse_cuda(e, "device query");
  if (major != 10 || minor != 3) return refuse(TSS_ERR_UNSUPPORTED_ARCH, "needs an sm_103 GPU");
  return TSS_OK;
}
// A workspace is its device's: kernels that use it are launched while that one is current.
inline tss_status still_on(int dev) {
  int now = -1;
  const cudaError_t e = cudaGetDevice(&now);
  if (e != cudaSuccess) return refuse_cuda(e, "device query");
  return now == dev ? TSS_OK : refuse(TSS_ERR_INVALID_ARG, "the current device is not the one that the workspace was made on");
}
// Device memory zeroed when this returns, whatever the calls that use it run on: a memset on the default stream would wait
// for that stream's work, and streams that do not synchronise with it would not wait for the memset.
inline cudaError_t zero_now(void* p, size_t bytes) {
  cudaStream_t s = nullptr;
  cudaError_t e = cudaStreamCreateWithFlags(&s, cudaStreamNonBlocking);
  if (e != cudaSuccess) return e;
  e = cudaMemsetAsync(p, 0, bytes, s);
  const cudaError_t done = cudaStreamSynchronize(s);
  cudaStreamDestroy(s);
  return e == cudaSuccess ? done : e;
}

// ------------------------------------------------------------------------------------------
// Vectors of N elements (N * element size a multiple of 4 bytes, addresses aligned to it) as fp32
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

template <int BYTES>
struct RawVec;
template <>
struct RawVec<8> { using type = uint2; };
template <>
struct RawVec<16> { using type = uint4; };

template <typename T, int N>
__device__ __forceinline__ void load_vec(const T* p, float* x) {
  constexpr int kPart = N * sizeof(T) < 16 ? N * sizeof(T) : 16;
  constexpr int kPer = kPart / sizeof(T);
#pragma unroll
  for (int i = 0; i < N / kPer; ++i) {
    const typename RawVec<kPart>::type raw = *reinterpret_cast<const typename RawVec<kPart>::type*>(p + i * kPer);
    T t[kPer];
    memcpy(t, &raw, kPart);
#pragma unroll
    for (int j = 0; j < kPer; ++j) x[i * kPer + j] = to_f32(t[j]);
  }
}
template <typename T, int N>
__device__ __forceinline__ void store_vec(T* p, const float* x) {
  constexpr int kPart = N * sizeof(T) < 16 ? N * sizeof(T) : 16;
  constexpr int kPer = kPart / sizeof(T);
#pragma unroll
  for (int i = 0; i < N / kPer; ++i) {
    T t[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) t[j] = from_f32<T>(x[i * kPer + j]);
    typename RawVec<kPart>::type raw;
    memcpy(&raw, t, kPart);
    *reinterpret_cast<typename RawVec<kPart>::type*>(p + i * kPer) = raw;
  }
}

// Eight elements as they lie in memory, and as fp32.
template <typename T>
struct Raw8 {
  uint4 v[8 * sizeof(T) / 16];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (size_t i = 0; i < sizeof(v) / 16; ++i) v[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (size_t i = 0; i < sizeof(v) / 16; ++i) v[i] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void to(float* x) const {
    T t[8];
    memcpy(t, v, sizeof(v));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_f32(t[i]);
  }
};

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z, w;\n\t"
      "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 w, x, y, z;\n\t"
      "mov.b64 {%0, %1}, w;\n\t}\n"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, w;\n\t"
      "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "add.rn.f32x2 w, x, y;\n\t"
      "mov.b64 {%0, %1}, w;\n\t}\n"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, w;\n\t"
      "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "mul.rn.f32x2 w, x, y;\n\t"
      "mov.b64 {%0, %1}, w;\n\t}\n"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

// The same on pairs kept in 64-bit registers (low half first), for loops where a pair is used often.
using f2_t = unsigned long long;
__device__ __forceinline__ f2_t f2_pack(float x, float y) {
  f2_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
  return v;
}
__device__ __forceinline__ float2 f2_unpack(f2_t v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}
__device__ __forceinline__ f2_t f2_fma(f2_t a, f2_t b, f2_t c) {
  f2_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ f2_t f2_mul(f2_t a, f2_t b) {
  f2_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ f2_t f2_add(f2_t a, f2_t b) {
  f2_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// ------------------------------------------------------------------------------------------
// A page of the 4-bit cache: one block per KV head (K codes, V codes, K parameters, V parameters;
// tss.h gives the order inside each)
// ------------------------------------------------------------------------------------------
constexpr int kPgTokens = TSS_PAGE_TOKENS;
constexpr int kPgGroup = 64;      // dims that share a scale and a minimum
constexpr int kPgMaxReq = 64;     // requests of a call
constexpr int kPgMaxRows = 128;   // rows of one request's block in the attention
template <int D>
struct PgBlock {
  static constexpr int kGroups = D / kPgGroup;
  static constexpr int kCodes = kPgTokens * D / 2;
  static constexpr int kK = 0, kV = kCodes, kKParams = 2 * kCodes;
  static constexpr int kParams = kPgTokens * kGroups * 4;
  static constexpr int kVParams = kKParams + kParams;
  static constexpr int kBytes = kVParams + kParams;
};
inline size_t pg_block_bytes(int head_dim) {
  return head_dim == 64 ? PgBlock<64>::kBytes : head_dim == 128 ? PgBlock<128>::kBytes : 0;
}

struct PgReq {
  int seq, first, n, row;  // sequence, first token, tokens, first row of the caller's arrays
};
struct PgBatch {
  int n_req;
  PgReq r[kPgMaxReq];
};

}  // namespace tss
