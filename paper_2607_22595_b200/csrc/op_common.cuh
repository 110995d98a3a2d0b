// What the operators without a context share: the message of a refused call, properties of the current device, and the
// loads of one row of router logits.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdarg.h>
#include <stdio.h>

#include <atomic>

#include "mix_internal.h"

namespace mix {

inline int op_fail(char* errbuf, int errbuf_len, int code, const char* fmt, ...) {
  if (errbuf && errbuf_len > 0) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(errbuf, (size_t)errbuf_len, fmt, ap);
    va_end(ap);
  }
  return code;
}
#define MIX_OP_FAIL(code, ...) return mix::op_fail(errbuf, errbuf_len, code, __VA_ARGS__)
#define MIX_OP_CUDA(expr)                                                                                        \
  do {                                                                                                           \
    const cudaError_t e_ = (expr);                                                                               \
    if (e_ != cudaSuccess) {                                                                                     \
      cudaGetLastError(); /* reported here, not left in the runtime's record */                                  \
      return mix::op_fail(errbuf, errbuf_len, MIX_ERR_CUDA, "%s: %s", #expr, cudaGetErrorString(e_));            \
    }                                                                                                            \
  } while (0)

// Index of the current device and its number of SMs (0, and the error, where there is none).
constexpr int kOpDevices = 64;
inline cudaError_t op_device(int* dev, int* n_sms) {
  static std::atomic<int> sms[kOpDevices];
  cudaError_t e = cudaGetDevice(dev);
  if (e != cudaSuccess) return e;
  if (*dev < 0 || *dev >= kOpDevices) return cudaErrorInvalidDevice;
  int n = sms[*dev].load(std::memory_order_relaxed);
  if (n == 0) {
    e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, *dev);
    if (e != cudaSuccess) return e;
    sms[*dev].store(n, std::memory_order_relaxed);
  }
  *n_sms = n;
  return cudaSuccess;
}

inline int op_elem_size(int dtype) { return dtype == MIX_DTYPE_F32 ? 4 : (dtype == MIX_DTYPE_BF16 || dtype == MIX_DTYPE_F16 ? 2 : 0); }

#ifdef __CUDACC__
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// A row of E router logits on G lanes (a power of two up to 32), V values a lane, in pieces of one 16-byte load: lane
// `sub` holds columns b * G * VW + sub * VW + i, i < VW, of every piece b.
template <typename T>
struct RowVec {
  static constexpr int VW = 16 / (int)sizeof(T);
};
template <typename T, int G>
__device__ __forceinline__ int row_col(int v, int sub) {
  constexpr int VW = RowVec<T>::VW;
  return (v / VW) * (G * VW) + sub * VW + v % VW;
}
// Columns behind the row's end and NaN read as -inf: no probability, never chosen.
template <typename T, int G, int V>
__device__ __forceinline__ void load_row(const T* __restrict__ row, int E, int sub, bool vec, float (&x)[V]) {
  constexpr int VW = RowVec<T>::VW;
  static_assert(V % VW == 0, "whole pieces");
#pragma unroll
  for (int b = 0; b < V / VW; ++b) {
    const int c0 = b * G * VW + sub * VW;
    if (vec && c0 + VW <= E) {
      const uint4 raw = *reinterpret_cast<const uint4*>(row + c0);
      const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
      for (int i = 0; i < VW; ++i) x[b * VW + i] = to_f32(e[i]);
    } else {
#pragma unroll
      for (int i = 0; i < VW; ++i) x[b * VW + i] = c0 + i < E ? to_f32(row[c0 + i]) : -INFINITY;
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) x[v] = x[v] == x[v] ? x[v] : -INFINITY;
}
template <typename T, int G, int V>
__device__ __forceinline__ void store_row(T* __restrict__ row, int E, int sub, bool vec, const float (&x)[V]) {
  constexpr int VW = RowVec<T>::VW;
#pragma unroll
  for (int b = 0; b < V / VW; ++b) {
    const int c0 = b * G * VW + sub * VW;
    if (vec && c0 + VW <= E) {
      uint4 raw;
      T* e = reinterpret_cast<T*>(&raw);
#pragma unroll
      for (int i = 0; i < VW; ++i) e[i] = from_f32<T>(x[b * VW + i]);
      *reinterpret_cast<uint4*>(row + c0) = raw;
    } else {
#pragma unroll
      for (int i = 0; i < VW; ++i)
        if (c0 + i < E) row[c0 + i] = from_f32<T>(x[b * VW + i]);
    }
  }
}

template <int G>
__device__ __forceinline__ float group_max(float x) {
#pragma unroll
  for (int o = 1; o < G; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
template <int G>
__device__ __forceinline__ float group_sum(float x) {
#pragma unroll
  for (int o = 1; o < G; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// Unnormalised score of a logit in a row whose largest is `top`.
//   softmax  e^(x - top); logits equal to the largest count 1 even where both are +inf -- the limit of equal logits that grow
//   sigmoid  sigmoid(x) e^-min(top, 0): where all logits of a row are low their sigmoids underflow together, their shares do not
__device__ __forceinline__ float score_softmax(float x, float top) { return x == -INFINITY ? 0.f : (x == top ? 1.f : expf(x - top)); }
__device__ __forceinline__ float score_sigmoid(float x, float top) {
  if (x == -INFINITY) return 0.f;
  return x > 0.f ? 1.f / (1.f + expf(-x)) : expf(x - fminf(top, 0.f)) / (1.f + expf(x));   // (x > 0: the largest is positive too)
}
__device__ __forceinline__ float score(int act, float x, float top) {
  return act == MIX_ACT_SOFTMAX ? score_softmax(x, top) : score_sigmoid(x, top);
}
__device__ __forceinline__ float sigmoidf(float x) { return 1.f / (1.f + expf(-x)); }
#endif

constexpr int kOpMaxExperts = 512;
constexpr int kOpMaxTopk = 16;

// Calls f(std::integral_constant<int, G>, std::integral_constant<int, V>) for the narrowest row layout that holds E columns.
#define MIX_ROW_LAYOUT(E, CALL)        \
  do {                                 \
    if ((E) <= 8) { CALL(1, 8); }      \
    else if ((E) <= 16) { CALL(2, 8); }\
    else if ((E) <= 32) { CALL(4, 8); }\
    else if ((E) <= 64) { CALL(8, 8); }\
    else if ((E) <= 128) { CALL(16, 8); }\
    else if ((E) <= 256) { CALL(32, 8); }\
    else { CALL(32, 16); }             \
  } while (0)

}  // namespace mix
