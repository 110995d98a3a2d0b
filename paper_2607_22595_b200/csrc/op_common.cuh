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
// Columns behind the row's end read as -inf: no probability, never chosen.
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
  if (G == 32) {
    float m;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(x));
    return m;
  }
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
// Does any lane of the group say yes?
template <int G>
__device__ __forceinline__ bool group_any(bool yes) {
  const unsigned votes = __ballot_sync(0xffffffffu, yes);
  const int first = (int)(threadIdx.x & 31) & ~(G - 1);
  return G == 32 ? votes != 0u : ((votes >> first) & ((1u << (G & 31)) - 1u)) != 0u;
}

// e^x as 2^(x log2 e) by the hardware's 2^x: the argument is off by half a step of itself (|x| U, U = 2^-24) and by what log2 e is off
// (0.22 |x| U), the result by two steps (4 U).  A logit's distance from the row's largest is rounded by as much already.  Results below
// 2^-126 are 0.  (65536 rows of 256 fp32, k = 8, with expf(x - top) instead: selection with the whole row's softmax 34.0 us, 32.5 so, its gradient
// 24.4, 23.2 so; balance loss of sigmoids 26.1 forward, 27.9 so, and 30.0 backward, 29.8 so.)
__device__ __forceinline__ float exp2_hw(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kLog2e = 1.44269502162933350f;
__device__ __forceinline__ float exp_row(float x) { return exp2_hw(x * kLog2e); }
// e^(x - top), with top log2 e at hand: one multiply-add, which rounds once.  What the rounding of top log2 e is off is a factor that
// all logits of the row have in common: within 2^(+-2^-8) up to |top| = 65536, whose product with log2 e is below 2^17.  Beyond, the
// factor would grow, and leave fp32's range from 1.4e9 on, so there the difference is taken first.  It is exact for every logit
// that has a score other than 0, one within 104 of such a top.
constexpr float kFarTop = 65536.f;
struct ExpFrom {
  float top, scaled;
  bool far;
  __device__ __forceinline__ explicit ExpFrom(float t) : top(t), scaled(t * kLog2e), far(fabsf(t) > kFarTop) {}
  __device__ __forceinline__ float operator()(float x) const { return far ? exp_row(x - top) : exp2_hw(fmaf(x, kLog2e, -scaled)); }
};
__device__ __forceinline__ float rcp_hw(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float sigmoid_row(float x) { return rcp_hw(1.f + exp_row(-x)); }

template <int V>
__device__ __forceinline__ float top_of(const float (&x)[V]) {             // (the larger of a NaN and a number is the number)
  float top = x[0];
#pragma unroll
  for (int v = 1; v < V; ++v) top = fmaxf(top, x[v]);
  return top;
}
// The score of one logit in a row whose largest is `top`; see scores().
__device__ __forceinline__ float score(int act, float x, float top) {
  if (x == -INFINITY) return 0.f;
  if (act == MIX_ACT_SOFTMAX) return top == INFINITY ? (x == top ? 1.f : 0.f) : ExpFrom(top)(x);
  return top >= 0.f ? sigmoid_row(x) : ExpFrom(top)(x) * rcp_hw(1.f + exp_row(x));
}
// Unnormalised scores of a lane's logits, in place, and their sum.  A NaN scores 0: one that is there makes the sum a NaN, which is
// looked at once for all V.
//   softmax  e^(x - top), `top` the row's largest logit.  Logits of +inf share the row, the limit of equal ones that grow: they
//            score 1, all others 0.
//   sigmoid  sigmoid(x).  Where all logits of a row are so low that their sigmoids underflow, their shares do not: `low` says
//            that the row's largest, below 0, is to be taken off, sigmoid(x) e^-top.
// slope: where given, score times (1 - sigmoid) of sigmoids, the score itself of a softmax
template <int V>
__device__ __forceinline__ float scores(int act, float top, bool low, float (&x)[V], float (*slope)[V] = nullptr) {
  float total = 0.f;
  if (act == MIX_ACT_SOFTMAX) {
    if (top == INFINITY) {
#pragma unroll
      for (int v = 0; v < V; ++v) x[v] = x[v] == INFINITY ? 0.f : -INFINITY;
      top = 0.f;
    } else if (top == -INFINITY) {
      top = 0.f;
    }
    const ExpFrom e(top);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      x[v] = e(x[v]);
      if (slope) (*slope)[v] = x[v];
      total += x[v];
    }
  } else if (!low) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float e = exp_row(-x[v]), s = rcp_hw(1.f + e);
      if (slope) (*slope)[v] = s * (fminf(e, 3e38f) * s);      // (where e is infinite s is 0)
      x[v] = s;
      total += s;
    }
  } else {
    const float off = top < 0.f && top > -INFINITY ? top : 0.f;
    const ExpFrom e(off);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float r = rcp_hw(1.f + exp_row(x[v])), s = off == 0.f ? sigmoid_row(x[v]) : e(x[v]) * r;
      if (slope) (*slope)[v] = s * r;
      x[v] = s;
      total += s;
    }
  }
  if (total != total) {
    total = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (x[v] != x[v]) {
        x[v] = 0.f;
        if (slope) (*slope)[v] = 0.f;
      }
      total += x[v];
    }
  }
  return total;
}
constexpr float kLowTotal = 1e-20f;        // below it a row's sigmoids are taken again with `low`
#endif

constexpr int kOpMaxExperts = 512;
constexpr int kOpMaxTopk = 16;
constexpr int kOpMaxRows = MIX_OP_MAX_ROWS;      // (row numbers and a grid's stride added to them stay in 31 bits)

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
