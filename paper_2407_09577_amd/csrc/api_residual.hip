// C ABI of the block residual and its gradients: argument checks and launches.
#include "flashnorm.h"
#include "fn_checks.h"
#include "fn_launch.h"

namespace {

struct Region {
  const void* p;
  int64_t bytes;
};

bool any_overlap(const Region& a, const Region* r, int n) {
  for (int i = 0; i < n; ++i)
    if (a.p && r[i].p && a.bytes > 0 && r[i].bytes > 0 && overlaps(a.p, a.bytes, r[i].p, r[i].bytes)) return true;
  return false;
}

// The checks both directions share: the inputs x, h, gate and the scalars.
int check_common(const fn::ResidualArgs& p, int64_t M, int64_t K, int64_t ldx, int64_t ldh, int64_t ldg,
                 int64_t gate_rows) {
  if (!dtype_ok(p.dtype)) return FN_ERR_DTYPE;
  if (M < 0 || K <= 0 || K % (p.dtype == FN_BF16 ? 8 : 4)) return FN_ERR_SHAPE;
  if (K > fn::kResidualMaxK) return FN_ERR_SIZE;
  int s;
  if ((s = check_matrix(p.x, M, K, ldx, p.dtype, true))) return s;
  if ((s = check_matrix(p.h, M, K, ldh, p.dtype, true))) return s;
  if (p.gate) {
    if (gate_rows < 1) return FN_ERR_SHAPE;
    if ((s = check_matrix(p.gate, M, K, ldg, p.dtype, true))) return s;
  }
  if (!aligned16(p.g_post) || !aligned16(p.g_pre)) return FN_ERR_ALIGN;
  if ((s = check_eps(p.eps_post)) || (s = check_eps(p.eps_pre))) return s;
  if (!isfinite(p.res_scale) || !isfinite(p.branch_scale)) return FN_ERR_VALUE;
  return FN_OK;
}

int64_t gates(int64_t M, int64_t gate_rows) { return (M + gate_rows - 1) / gate_rows; }

}  // namespace

extern "C" {

int flashnorm_block_residual(const void* x, int64_t ldx, const void* h, int64_t ldh, int64_t M, int64_t K, int dtype,
                             const float* g_post, float eps_post, const void* gate, int64_t ldg, int64_t rows_per_gate,
                             float res_scale, float branch_scale, const float* g_pre, float eps_pre, void* out,
                             int64_t ldo, void* normed, int64_t ldn, float* inv_rms, void* stream) {
  fn::ResidualArgs p{};
  p.x = x, p.h = h, p.gate = gate, p.dtype = dtype;
  p.g_post = g_post, p.g_pre = g_pre, p.eps_post = eps_post, p.eps_pre = eps_pre;
  p.res_scale = res_scale, p.branch_scale = branch_scale;
  int s = check_common(p, M, K, ldx, ldh, ldg, rows_per_gate);
  if (s) return s;
  if ((s = check_matrix(out, M, K, ldo, dtype, true))) return s;
  if (normed) {
    if (!g_pre) return FN_ERR_NULL;
    if ((s = check_matrix(normed, M, K, ldn, dtype, true))) return s;
  }
  if (reinterpret_cast<uintptr_t>(inv_rms) % 4) return FN_ERR_ALIGN;
  if (M == 0) return FN_OK;
  if (rows_per_gate > M) rows_per_gate = M;
  const Region X{x, extent_bytes(M, K, ldx, dtype)}, H{h, extent_bytes(M, K, ldh, dtype)};
  const Region G{gate, gate ? extent_bytes(gates(M, rows_per_gate), K, ldg, dtype) : 0};
  const Region GP{g_post, K * 4}, GN{g_pre, K * 4};
  const Region O{out, extent_bytes(M, K, ldo, dtype)}, NO{normed, extent_bytes(M, K, ldn, dtype)}, R{inv_rms, M * 4};
  // Each element is read before it is written, by the same thread: out may be h, normed may be x.
  const bool out_is_h = out == h && ldo == ldh, normed_is_x = normed == x && ldn == ldx;
  const Region out_in[] = {X, G, GP, GN, NO, R, out_is_h ? Region{nullptr, 0} : H};
  const Region norm_in[] = {H, G, GP, GN, R, normed_is_x ? Region{nullptr, 0} : X};
  const Region rms_in[] = {X, H, G, GP, GN};
  if (any_overlap(O, out_in, 7) || any_overlap(NO, norm_in, 6) || any_overlap(R, rms_in, 5)) return FN_ERR_ALIAS;
  p.M = (int)M, p.K = (int)K, p.ldx = (int)ldx, p.ldh = (int)ldh, p.ldg = (int)ldg;
  p.gate_rows = gate ? (int)rows_per_gate : 1;
  p.out = out, p.normed = normed, p.ldo = (int)ldo, p.ldn = (int)ldn, p.inv_rms = inv_rms;
  p.stream = (hipStream_t)stream;
  return status_of(fn::launch_residual(p));
}

size_t flashnorm_block_residual_bwd_size(int64_t M, int64_t K, int64_t rows_per_gate, int dtype) {
  if (!dtype_ok(dtype) || M < 0 || M > kMaxRows || K <= 0 || K > fn::kResidualMaxK ||
      K % (dtype == FN_BF16 ? 8 : 4) || rows_per_gate < 0)
    return 0;
  if (M == 0) return 16;
  return 4 * (size_t)fn::residual_bwd_ws_floats(M, K, rows_per_gate < 1 ? 1 : rows_per_gate > M ? M : rows_per_gate,
                                                dtype, true, true, rows_per_gate > 0);
}

int flashnorm_block_residual_bwd(const void* x, int64_t ldx, const void* h, int64_t ldh, const void* dh_out,
                                 int64_t lddo, const void* dn, int64_t lddn, int64_t M, int64_t K, int dtype,
                                 const float* g_post, float eps_post, const void* gate, int64_t ldg,
                                 int64_t rows_per_gate, float res_scale, float branch_scale, const float* g_pre,
                                 float eps_pre, void* dx, int64_t lddx, void* dh, int64_t lddh, void* dgate,
                                 int64_t lddg, float* dg_post, float* dg_pre, void* workspace, size_t workspace_bytes,
                                 void* stream) {
  fn::ResidualArgs p{};
  p.x = x, p.h = h, p.gate = gate, p.dtype = dtype;
  p.g_post = g_post, p.g_pre = g_pre, p.eps_post = eps_post, p.eps_pre = eps_pre;
  p.res_scale = res_scale, p.branch_scale = branch_scale;
  int s = check_common(p, M, K, ldx, ldh, ldg, rows_per_gate);
  if (s) return s;
  if (M > 0 && ((!dh_out && !dn) || (g_pre && !dn))) return FN_ERR_NULL;
  if (dn && !g_pre) return FN_ERR_NULL;
  if (dh_out && (s = check_matrix(dh_out, M, K, lddo, dtype, true))) return s;
  if (dn && (s = check_matrix(dn, M, K, lddn, dtype, true))) return s;
  if ((s = check_matrix(dx, M, K, lddx, dtype, true))) return s;
  if ((s = check_matrix(dh, M, K, lddh, dtype, true))) return s;
  if ((dgate && !gate) || (dg_post && !g_post) || (dg_pre && !g_pre)) return FN_ERR_NULL;
  if (dgate && (s = check_matrix(dgate, M, K, lddg, dtype, true))) return s;
  if (!aligned16(dg_post) || !aligned16(dg_pre) || !aligned16(workspace)) return FN_ERR_ALIGN;
  if (M > 0 && rows_per_gate > M) rows_per_gate = M;
  const int64_t T = gate ? rows_per_gate : 1, B = gate ? gates(M, T) : 0;
  const int64_t need = M ? 4 * fn::residual_bwd_ws_floats(M, K, T, dtype, dg_post, dg_pre, dgate) : 0;
  if (need && !workspace) return FN_ERR_NULL;
  if ((uint64_t)need > workspace_bytes) return FN_ERR_SIZE;
  const int64_t mk = K * elem_size(dtype);
  auto mat = [&](const void* q, int64_t rows, int64_t ld) {
    return Region{q, q && rows > 0 ? (rows - 1) * ld * elem_size(dtype) + mk : 0};
  };
  const Region in[] = {mat(x, M, ldx),    mat(h, M, ldh),      mat(dh_out, M, lddo),
                       mat(dn, M, lddn),  mat(gate, B, ldg),   Region{g_post, g_post ? K * 4 : 0},
                       Region{g_pre, g_pre ? K * 4 : 0}};
  const Region outs[] = {mat(dx, M, lddx), mat(dh, M, lddh), mat(dgate, B, lddg), Region{dg_post, dg_post ? K * 4 : 0},
                         Region{dg_pre, dg_pre ? K * 4 : 0}, Region{workspace, need}};
  for (int i = 0; i < 6; ++i)
    if (any_overlap(outs[i], in, 7) || any_overlap(outs[i], outs + i + 1, 5 - i)) return FN_ERR_ALIAS;
  p.M = (int)M, p.K = (int)K, p.ldx = (int)ldx, p.ldh = (int)ldh, p.ldg = (int)ldg, p.gate_rows = (int)T;
  p.dh_out = dh_out, p.dn = dn, p.lddo = (int)lddo, p.lddn = (int)lddn;
  p.dx = dx, p.dh = dh, p.dgate = dgate, p.lddx = (int)lddx, p.lddh = (int)lddh, p.lddg = (int)lddg;
  p.dg_post = dg_post, p.dg_pre = dg_pre, p.ws = (float*)workspace;
  p.stream = (hipStream_t)stream;
  if (M == 0 && !dg_post && !dg_pre) return FN_OK;
  return status_of(fn::launch_residual_bwd(p));
}

}  // extern "C"
