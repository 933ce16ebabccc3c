// Reading a weight view of any strides for the folds.
#pragma once

#include "fn_device.h"

namespace fn {

// Packed column -> logical column, or -1 for padding.
__device__ __forceinline__ int64_t logical_col(int64_t p, int64_t N, int glu) {
  if (!glu) return p < N ? p : -1;
  const int64_t F = N / 2;
  const int64_t pair = p / 32, within = p % 32;
  const int64_t f = pair * 16 + (within & 15);
  if (f >= F) return -1;
  return within < 16 ? f : F + f;
}

__device__ __forceinline__ float widen(unsigned short b) { return __uint_as_float((unsigned)b << 16); }
__device__ __forceinline__ float widen(float f) { return f; }

// Eight consecutive k of logical column n (zeros past K or without a column).  vec: the k are
// contiguous, K is a multiple of 8 and every such run starts on 16 bytes.  The addresses are
// clamped and the values selected, so that no load stands behind a branch and the loads of
// several fragments are in flight together.
template <typename T>
__device__ __forceinline__ void load_k8(const T* __restrict__ W, int64_t sk, int64_t sn, int64_t k0, int64_t n,
                                        int64_t K, bool vec, float (&w)[8]) {
  const int64_t nc = n >= 0 ? n : 0;
  if (vec) {
    const bool ok = n >= 0 && k0 < K;
    const T* p = W + nc * sn + (k0 < K ? k0 : 0);
    if constexpr (sizeof(T) == 2) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[2 * i] = ok ? bf16_lo(v[i]) : 0.0f, w[2 * i + 1] = ok ? bf16_hi(v[i]) : 0.0f;
    } else {
      const f32x4 v0 = *reinterpret_cast<const f32x4*>(p), v1 = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = ok ? v0[i] : 0.0f, w[4 + i] = ok ? v1[i] : 0.0f;
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int64_t k = k0 + e;
    const float v = widen(W[(k < K ? k : 0) * sk + nc * sn]);
    w[e] = n >= 0 && k < K ? v : 0.0f;
  }
}

// Eight consecutive values of an optional vector over K (`none` without one, or past K).
__device__ __forceinline__ void load_v8(const float* __restrict__ v, int64_t k0, int64_t K, bool vec, float none,
                                        float (&x)[8]) {
  if (v && vec && k0 + 8 <= K) {
    const f32x4 v0 = *reinterpret_cast<const f32x4*>(v + k0), v1 = *reinterpret_cast<const f32x4*>(v + k0 + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v0[i], x[4 + i] = v1[i];
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = v && k0 + e < K ? v[k0 + e] : none;
}

}  // namespace fn
