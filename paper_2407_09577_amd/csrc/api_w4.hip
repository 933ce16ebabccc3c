// C ABI of the 4-bit weights and their products: argument checks and launches.
#include "flashnorm.h"
#include "fn_checks.h"
#include "fn_launch.h"

namespace {

using fn::EpiArgs;

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }

// Geometry of a packed 4-bit weight.
int check_w4(int64_t K, int64_t N, int layout, int group) {
  if (layout != FN_LAYOUT_LINEAR && layout != FN_LAYOUT_GLU) return FN_ERR_VALUE;
  if (!group_ok(group)) return FN_ERR_VALUE;
  if (K <= 0 || N <= 0 || (layout == FN_LAYOUT_GLU && N % 2)) return FN_ERR_SHAPE;
  if (K > kMaxLd || N > kMaxRows || fn::w4_bytes(K, N, layout == FN_LAYOUT_GLU, group) > kMaxPackedBytes)
    return FN_ERR_SIZE;
  return FN_OK;
}

int64_t w4_groups(int64_t K, int group) { return (K + group - 1) / group; }

struct W4Op {
  const void* a;
  int64_t M, K, lda;
  int a_dtype;
  const float* g;
  const void* w4;
  int64_t ncols;  // N, or F for a GLU
  int glu, group;
  void* y;
  int64_t ldy;
  int y_dtype;
  int epi;
  float eps;
  const float* bias;
  float* inv_rms;
  const float* row_scale;
  void* ws;
  size_t ws_bytes;
  void* stream;
};

int run_w4(const W4Op& d) {
  if (!dtype_ok(d.a_dtype) || d.a_dtype != d.y_dtype) return FN_ERR_DTYPE;
  if (d.a_dtype != FN_BF16) return FN_ERR_UNSUPPORTED;
  const int64_t N = d.glu ? 2 * d.ncols : d.ncols;
  if (d.ncols <= 0 || d.ncols > kMaxRows) return FN_ERR_SHAPE;
  int s = check_w4(d.K, N, d.glu ? FN_LAYOUT_GLU : FN_LAYOUT_LINEAR, d.group);
  if (s) return s;
  if (d.K % 8) return FN_ERR_SHAPE;
  if ((s = check_matrix(d.a, d.M, d.K, d.lda, d.a_dtype, true))) return s;
  if ((s = check_matrix(d.y, d.M, d.ncols, d.ldy, d.y_dtype, true))) return s;
  if (!d.w4) return FN_ERR_NULL;
  if (!aligned16(d.w4) || !aligned16(d.g) || !aligned16(d.bias) || !aligned4(d.inv_rms) || !aligned4(d.row_scale))
    return FN_ERR_ALIGN;
  if ((s = check_eps(d.eps))) return s;
  if (d.M == 0) return FN_OK;
  const int64_t ybytes = extent_bytes(d.M, d.ncols, d.ldy, d.y_dtype);
  const int64_t wbytes = fn::w4_bytes(d.K, N, d.glu, d.group);
  if (overlaps(d.y, ybytes, d.a, extent_bytes(d.M, d.K, d.lda, d.a_dtype)) || overlaps(d.y, ybytes, d.w4, wbytes) ||
      (d.g && overlaps(d.y, ybytes, d.g, d.K * 4)) || (d.bias && overlaps(d.y, ybytes, d.bias, d.ncols * 4)) ||
      (d.row_scale && overlaps(d.y, ybytes, d.row_scale, d.M * 4)))
    return FN_ERR_ALIAS;
  if (d.inv_rms) {
    const int64_t rbytes = d.M * 4;
    if (overlaps(d.inv_rms, rbytes, d.y, ybytes) ||
        overlaps(d.inv_rms, rbytes, d.a, extent_bytes(d.M, d.K, d.lda, d.a_dtype)) ||
        overlaps(d.inv_rms, rbytes, d.w4, wbytes) || (d.g && overlaps(d.inv_rms, rbytes, d.g, d.K * 4)) ||
        (d.bias && overlaps(d.inv_rms, rbytes, d.bias, d.ncols * 4)))
      return FN_ERR_ALIAS;
  }
  const int64_t NP = fn::packed_cols(N, d.glu), KB = fn::w4_blocks(d.K);
  const fn::W4Plan plan = fn::w4_plan((int)d.M, (int)d.K, (int)KB, (int)NP, d.glu, d.group, d.g != nullptr);
  const int64_t need = fn::w4_workspace(plan, d.M, KB, NP);
  if (need > 0) {
    if (!d.ws) return FN_ERR_NULL;
    if (!aligned16(d.ws)) return FN_ERR_ALIGN;
    if ((uint64_t)need > d.ws_bytes) return FN_ERR_SIZE;
    if (overlaps(d.ws, need, d.y, ybytes) || overlaps(d.ws, need, d.a, extent_bytes(d.M, d.K, d.lda, d.a_dtype)) ||
        overlaps(d.ws, need, d.w4, wbytes) || (d.g && overlaps(d.ws, need, d.g, d.K * 4)) ||
        (d.bias && overlaps(d.ws, need, d.bias, d.ncols * 4)) ||
        (d.row_scale && overlaps(d.ws, need, d.row_scale, d.M * 4)) ||
        (d.inv_rms && overlaps(d.ws, need, d.inv_rms, d.M * 4)))
      return FN_ERR_ALIAS;
  }
  EpiArgs ep{};
  ep.eps = d.eps;
  ep.inv_k = 1.0f / (float)d.K;
  ep.inv_kd = 1.0 / (double)d.K;
  ep.bias = d.bias;
  ep.inv_rms = d.inv_rms;
  ep.row_scale = d.row_scale;
  ep.g_rt = d.g;
  fn::W4Args p{(const __bf16*)d.a, (int)d.M, (int)d.K, (int)d.lda, d.w4,
               fn::w4_scales(const_cast<void*>(d.w4), d.K, N, d.glu),
               fn::w4_norms(const_cast<void*>(d.w4), d.K, N, d.glu, d.group), (int)NP, (int)KB, d.group,
               (int)d.ncols, (__bf16*)d.y, (int)d.ldy, d.epi, ep, plan, d.ws, (hipStream_t)d.stream};
  const hipError_t e = fn::launch_w4(p);
  return e == hipErrorInvalidConfiguration ? FN_ERR_SIZE : status_of(e);
}

}  // namespace

extern "C" {

size_t fold_weights_w4_size(int64_t K, int64_t N, int layout, int group) {
  return check_w4(K, N, layout, group) ? 0 : (size_t)fn::w4_bytes(K, N, layout == FN_LAYOUT_GLU, group);
}

int fold_weights_w4(const void* W, int64_t stride_k, int64_t stride_n, int w_dtype, const float* g, int64_t K, int64_t N,
                    int layout, int group, int zero_points, void* W4, void* stream) {
  if (!dtype_ok(w_dtype)) return FN_ERR_DTYPE;
  int s = check_w4(K, N, layout, group);
  if (s) return s;
  if (zero_points != 0 && zero_points != 1) return FN_ERR_VALUE;
  if (stride_k < 0 || stride_n < 0) return FN_ERR_SHAPE;
  if (stride_k >= kMaxFoldStrideK || stride_n >= kMaxFoldStrideN) return FN_ERR_SIZE;
  if (!W || !W4) return FN_ERR_NULL;
  if (!aligned16(W4) || reinterpret_cast<uintptr_t>(W) % elem_size(w_dtype)) return FN_ERR_ALIGN;
  const int64_t wb = fn::w4_bytes(K, N, layout == FN_LAYOUT_GLU, group);
  const int64_t wext = view_bytes(K, N, stride_k, stride_n, w_dtype);
  if (overlaps(W4, wb, W, wext) || (g && overlaps(W4, wb, g, K * 4))) return FN_ERR_ALIAS;
  fn::W4FoldArgs p{W, stride_k, stride_n, w_dtype, g, K, N, layout == FN_LAYOUT_GLU, group, zero_points != 0, W4,
                   (hipStream_t)stream};
  return status_of(fn::launch_w4_fold(p));
}

int pack_weights_w4(const uint8_t* codes, int64_t ldc, const float* scales, int64_t lds, const uint8_t* zeros,
                    int64_t ldz, int64_t K, int64_t N, int layout, int group, void* W4, void* stream) {
  int s = check_w4(K, N, layout, group);
  if (s) return s;
  if (ldc < N || lds < N || (zeros && ldz < N)) return FN_ERR_SHAPE;
  if (ldc >= kMaxFoldStrideK || lds >= kMaxFoldStrideK || (zeros && ldz >= kMaxFoldStrideK)) return FN_ERR_SIZE;
  if (!codes || !scales || !W4) return FN_ERR_NULL;
  if (!aligned16(W4) || reinterpret_cast<uintptr_t>(scales) % 4) return FN_ERR_ALIGN;
  const int64_t wb = fn::w4_bytes(K, N, layout == FN_LAYOUT_GLU, group), G = w4_groups(K, group);
  if (overlaps(W4, wb, codes, (K - 1) * ldc + N) || overlaps(W4, wb, scales, ((G - 1) * lds + N) * 4) ||
      (zeros && overlaps(W4, wb, zeros, (G - 1) * ldz + N)))
    return FN_ERR_ALIAS;
  return status_of(fn::launch_w4_pack(codes, ldc, scales, lds, zeros, ldz, K, N, layout == FN_LAYOUT_GLU, group, W4,
                                      (hipStream_t)stream));
}

int unpack_weights_w4(const void* W4, int64_t K, int64_t N, int layout, int group, float* out, int64_t ldo,
                      void* stream) {
  int s = check_w4(K, N, layout, group);
  if (s) return s;
  if (ldo < N) return FN_ERR_SHAPE;
  if (ldo >= kMaxFoldStrideK) return FN_ERR_SIZE;
  if (!W4 || !out) return FN_ERR_NULL;
  if (!aligned16(W4) || reinterpret_cast<uintptr_t>(out) % 4) return FN_ERR_ALIGN;
  if (overlaps(out, extent_bytes(K, N, ldo, FN_F32), W4, fn::w4_bytes(K, N, layout == FN_LAYOUT_GLU, group)))
    return FN_ERR_ALIAS;
  return status_of(fn::launch_w4_unpack(W4, K, N, layout == FN_LAYOUT_GLU, group, out, ldo, (hipStream_t)stream));
}

size_t flashnorm_w4_workspace_size(int64_t M, int64_t K, int64_t N, int layout, int group) {
  if (M < 0 || M > kMaxRows || check_w4(K, N, layout, group)) return 0;
  const bool glu = layout == FN_LAYOUT_GLU;
  return (size_t)fn::w4_workspace(M, K, fn::packed_cols(N, glu), glu, group);
}

int flashnorm_linear_w4(const void* a, int64_t M, int64_t K, int64_t lda, int a_dtype, const float* g, const void* W4,
                        int64_t N, int group, float eps, const float* bias, void* y, int64_t ldy, int y_dtype,
                        float* inv_rms, void* workspace, size_t workspace_bytes, void* stream) {
  return run_w4(W4Op{a, M, K, lda, a_dtype, g, W4, N, 0, group, y, ldy, y_dtype, fn::EPI_RMS, eps, bias, inv_rms,
                     nullptr, workspace, workspace_bytes, stream});
}

int flashnorm_glu_w4(const void* a, int64_t M, int64_t K, int64_t lda, int a_dtype, const float* g, const void* W4_gu,
                     int64_t F, int group, float eps, void* out, int64_t ldo, int out_dtype, void* workspace,
                     size_t workspace_bytes, void* stream) {
  return run_w4(W4Op{a, M, K, lda, a_dtype, g, W4_gu, F, 1, group, out, ldo, out_dtype, fn::EPI_GLU, eps, nullptr,
                     nullptr, nullptr, workspace, workspace_bytes, stream});
}

int rowscale_linear_w4(const void* x, int64_t M, int64_t K, int64_t ldx, int x_dtype, const void* W4, int64_t N,
                       int group, const float* row_scale, void* y, int64_t ldy, int y_dtype, void* workspace,
                       size_t workspace_bytes, void* stream) {
  return run_w4(W4Op{x, M, K, ldx, x_dtype, nullptr, W4, N, 0, group, y, ldy, y_dtype, fn::EPI_ROWSCALE, 0.0f, nullptr,
                     nullptr, row_scale, workspace, workspace_bytes, stream});
}

}  // extern "C"
