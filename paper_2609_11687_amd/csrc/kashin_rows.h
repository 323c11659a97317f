// Rows of activations: element types, and loads and stores of eight consecutive entries as fp32 (used by
// the norm and the products from the codes).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstring>

#include "kashin.h"

namespace kashin {
namespace {

struct e4m3_t {
  uint8_t bits;
};

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(_Float16 v) { return static_cast<float>(v); }
__device__ __forceinline__ float widen(__bf16 v) { return static_cast<float>(v); }
__device__ __forceinline__ float widen(e4m3_t v) { return __builtin_amdgcn_cvt_f32_fp8(v.bits, 0); }

// Entries p[0 .. 7], those from `valid` on as zero.  The eight are read with one or two vector loads whatever the
// row's alignment (global memory takes unaligned vectors); only a row's last, partial eight is read
// entry by entry.
template <class T>
__device__ __forceinline__ void load8(const T* p, int valid, float (&v)[8]) {
  if (valid >= 8) {
    T q[8];
    __builtin_memcpy(q, p, sizeof(q));
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = widen(q[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < valid ? widen(p[j]) : 0.f;
  }
}

// Rounded to the nearest T (ties to even), as load8.
template <class T>
__device__ __forceinline__ void store8(T* p, int valid, const float (&v)[8]) {
  if (valid >= 8) {
    T q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = static_cast<T>(v[j]);
    __builtin_memcpy(p, q, sizeof(q));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < valid) p[j] = static_cast<T>(v[j]);
  }
}
// e4m3 of values within +-448 (the conversion gives NaN beyond)
__device__ __forceinline__ void store8(e4m3_t* p, int valid, const float (&v)[8]) {
  uint32_t q[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * k], v[4 * k + 1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * k + 2], v[4 * k + 3], w, true);
    q[k] = static_cast<uint32_t>(w);
  }
  if (valid >= 8) {
    __builtin_memcpy(p, q, sizeof(q));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < valid) p[j].bits = static_cast<uint8_t>(q[j / 4] >> (8 * (j % 4)));
  }
}

template <class T>
__device__ __forceinline__ void put4_as(T* y, int64_t valid, const float (&v)[4]) {
  T q[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) q[j] = static_cast<T>(v[j]);
  if (valid >= 4) {
    __builtin_memcpy(y, q, sizeof(q));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < valid) y[j] = q[j];
  }
}
// Four entries of KASHIN_F32, _F16 or _BF16 rows from i on, of which `valid` exist.
__device__ __forceinline__ void put4(void* y, int dtype, int64_t i, int64_t valid, const float (&v)[4]) {
  if (dtype == KASHIN_F32) put4_as(static_cast<float*>(y) + i, valid, v);
  else if (dtype == KASHIN_F16) put4_as(static_cast<_Float16*>(y) + i, valid, v);
  else put4_as(static_cast<__bf16*>(y) + i, valid, v);
}

// f(T()) for the element type of a KASHIN_F32 / _F16 / _BF16 code (checked by the caller)
template <class F>
auto with_float_type(int dtype, F&& f) {
  if (dtype == KASHIN_F32) return f(float());
  if (dtype == KASHIN_F16) return f(_Float16());
  return f(__bf16());
}

}  // namespace
}  // namespace kashin
