// Argument checks shared by the C ABI's files (host only).
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "flashnorm.h"
#include "fn_launch.h"

namespace {

constexpr int64_t kMaxLd = int64_t(1) << 21;    // leading dimensions, K (keeps tile extents < 2^31)
constexpr int64_t kMaxRows = int64_t(1) << 30;  // M, N
// Packed weight buffer: the matrix-core kernels address it with 32-bit byte
// offsets and use offsets >= 2^31 as out-of-range (zero-returning) loads.
constexpr int64_t kMaxPackedBytes = (int64_t(1) << 31) - 1;
// Strides of the weight view fold_weights reads: with K <= 2^21 and N <= 2^30 every
// element offset stays below 2^62.
constexpr int64_t kMaxFoldStrideK = int64_t(1) << 40;
constexpr int64_t kMaxFoldStrideN = int64_t(1) << 31;

inline int64_t packed_bytes(int64_t K, int64_t N, bool glu, int64_t elem) {
  return fn::packed_rows(K) * fn::packed_cols(N, glu) * elem;
}

inline bool dtype_ok(int d) { return d == FN_F32 || d == FN_BF16; }
inline int64_t elem_size(int d) { return d == FN_BF16 ? 2 : 4; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int64_t row_align(int d) { return 16 / elem_size(d); }

inline bool overlaps(const void* p, int64_t pbytes, const void* q, int64_t qbytes) {
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(p), b0 = reinterpret_cast<uintptr_t>(q);
  return a0 < b0 + (uintptr_t)qbytes && b0 < a0 + (uintptr_t)pbytes;
}

inline int64_t extent_bytes(int64_t rows, int64_t cols, int64_t ld, int dtype) {
  return rows > 0 ? ((rows - 1) * ld + cols) * elem_size(dtype) : 0;
}

// Bytes spanned by a strided view.  The largest element offset is below 2^62, its bytes may pass 2^63: they are counted
// without a sign, as overlaps() does.
inline int64_t view_bytes(int64_t K, int64_t N, int64_t stride_k, int64_t stride_n, int dtype) {
  return (int64_t)((uint64_t)((K - 1) * stride_k + (N - 1) * stride_n + 1) * (uint64_t)elem_size(dtype));
}

// Common checks of an activation-like operand [M, K] with leading dimension ld.
inline int check_matrix(const void* p, int64_t M, int64_t K, int64_t ld, int dtype, bool required) {
  if (M < 0 || K <= 0 || M > kMaxRows) return FN_ERR_SHAPE;
  if (ld < K) return FN_ERR_SHAPE;
  if (ld > kMaxLd) return FN_ERR_SIZE;
  if (required && M > 0 && !p) return FN_ERR_NULL;
  if (!aligned16(p) || ld % row_align(dtype)) return FN_ERR_ALIGN;
  return FN_OK;
}

inline int check_eps(float eps) { return (isfinite(eps) && eps >= 0.0f) ? FN_OK : FN_ERR_VALUE; }

inline int status_of(hipError_t e) { return e == hipSuccess ? FN_OK : FN_ERR_HIP; }

}  // namespace
