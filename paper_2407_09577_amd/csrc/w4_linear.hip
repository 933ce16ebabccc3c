// Products with 4-bit weights: which kernel and workgroup shape of w4_kernels.h a call takes, and its launches.
#include "flashnorm.h"
#include "w4_kernels.h"

namespace fn {

extern template hipError_t launch_w4_few<EPI_RMS>(const W4Args&, int);
extern template hipError_t launch_w4_few<EPI_GLU>(const W4Args&, int);
extern template hipError_t launch_w4_few<EPI_ROWSCALE>(const W4Args&, int);
extern template hipError_t launch_w4_many<EPI_RMS>(const W4Gemm&, int, int, hipStream_t);
extern template hipError_t launch_w4_many<EPI_GLU>(const W4Gemm&, int, int, hipStream_t);
extern template hipError_t launch_w4_many<EPI_ROWSCALE>(const W4Gemm&, int, int, hipStream_t);

// Workgroup shapes: rows, packed columns, k groups, workgroups that a compute unit holds, and the time in us
// on MI355X of w workgroups whose waves walk `sets` sets, r = w / 256 the workgroups per compute unit:
//   start ceil(r / per_cu) + sets (full (ceil(r / per_cu) - 1) + last) + each r,
// `last` going from one to full as the last round fills up.  Beside it stand what the kernel's launches cost
// (kW4FewUs, kW4ManyUs), the activations' pass and, with splits of K, the join of their sums.  The constants
// are least-squares fits over 900 (few rows: 1..256 rows) and 500 (17..2048 rows) random shapes of K 256..11008
// and 256..22016 columns, linear and GLU, groups of 128, each shape's weights read in turn from 400 MB: 5%
// rms for the many-row shapes and 8 to 12% for the few-row ones, whose times are launches in large part.  The
// shape so chosen took 0.8% (many rows) and 1.7 to 2.8% (few) more than the best of each call, in the mean.
// One workgroup of four waves leaves a compute unit's SIMDs a wave each, which neither hides its reads nor its
// widening: where a call has no more than a workgroup for each, two or eight k groups do (695 x 3928 x 3520:
// 42.4 us with 96 x 128 tiles, 35.2 with two k groups on each).  Two blocks of rows on a few-row workgroup widen the
// codes once for both, where the width alone fills the chip (32 x 4096 -> 22016 GLU: 21.5 us with one, 18.6 with two).
// The few-row kernel is not for few rows alone: narrow products of many rows take it too, which spares them the pass over
// the rows and the join (500 x 1024 -> 1024 9.3 -> 5.9 us, 432 x 5720 -> 284 16.5 -> 10.5, 1269 x 2328 -> 384
// 14.0 -> 9.6).
struct W4Shape {
  int rows, cols, ks, per_cu;
  float start, full, one, each;
};
static constexpr W4Shape kW4Few[] = {
    {16, 32, 8, 2, 0.586f, 1.376f, 0.630f, 0.0f},   {16, 64, 8, 2, 0.390f, 2.886f, 1.144f, 0.315f},
    {16, 96, 8, 2, 0.083f, 4.234f, 1.640f, 0.719f}, {16, 64, 4, 4, 0.522f, 2.440f, 0.829f, 0.137f},
    {16, 32, 4, 4, 0.781f, 1.411f, 0.502f, 0.0f},   {32, 64, 8, 1, 0.0f, 2.426f, 1.812f, 0.912f},
    {32, 96, 8, 1, 0.244f, 3.002f, 2.480f, 1.539f}, {16, 16, 8, 2, 0.817f, 0.751f, 0.411f, 0.0f},
    {16, 16, 16, 1, 0.502f, 0.684f, 0.890f, 0.0f},  {16, 48, 8, 2, 0.733f, 1.826f, 0.826f, 0.0f}};
static constexpr W4Shape kW4Many[] = {
    {128, 256, 1, 2, 3.165f, 3.130f, 1.989f, 1.234f}, {128, 128, 1, 2, 0.875f, 1.652f, 1.123f, 2.066f},
    {96, 256, 1, 2, 2.034f, 2.360f, 1.570f, 1.851f},  {96, 128, 1, 3, 0.747f, 1.858f, 0.905f, 1.419f},
    {64, 128, 2, 2, 0.282f, 1.972f, 1.184f, 1.612f},  {64, 128, 1, 4, 0.235f, 1.875f, 0.705f, 1.036f},
    {32, 128, 2, 4, 0.0f, 2.838f, 0.858f, 1.003f},    {32, 64, 4, 2, 0.099f, 1.609f, 0.953f, 0.838f},
    {96, 128, 2, 1, 0.910f, 1.486f, 1.410f, 2.521f},  {128, 128, 2, 1, 1.384f, 1.805f, 1.742f, 2.935f},
    {32, 32, 8, 1, 0.217f, 1.577f, 1.160f, 1.203f}};
constexpr int kW4FewLinearOnly = 7;  // from here on: an odd number of column blocks holds no gate/up pairs
constexpr float kW4FewUs = 4.15f, kW4FewPerMK = 0.915f;
constexpr float kW4ManyUs = 7.14f, kW4ManyPerMK = 0.859f, kW4JoinUs = 3.04f, kW4JoinPerMB = 0.255f;

// A non-negative x rounded up (ceilf would be a call).
static float up(float x) {
  const float t = (float)(int64_t)x;
  return t < x ? t + 1.0f : t;
}

static float shape_us(const W4Shape& s, int64_t wgs, int sets) {
  const float r = (float)wgs / 256.0f, rounds = up(r / s.per_cu);
  const float in_last = up(r - (rounds - 1.0f) * s.per_cu);
  const float fill = s.per_cu > 1 ? (in_last - 1.0f) / (s.per_cu - 1) : 0.0f;
  return s.start * rounds + sets * (s.full * (rounds - 1.0f) + s.one + (s.full - s.one) * fill) + s.each * r;
}

// The least time of each kernel, and how (NP and KB: packed columns and k blocks).
struct W4Best {
  W4Plan plan;
  float us;
};

// Smaller groups and a run-time g cost the few-row kernel most: a scale, a sum and four multiply-adds per group and
// column, and two matrix-core operations for one.  Measured at 150..1269 rows as factors of the shapes' times (1.35 to 1.6
// for groups of 32, 1.15 to 1.25 for 64; with g 1.4 to 1.9).
static W4Best few_plan(int M, int K, int KB, int NP, bool glu, int group, bool gs) {
  W4Best best{{false, 0, 1, KB}, 1e30f};
  const float x = (group == 32 ? 1.45f : group == 64 ? 1.18f : 1.0f) * (gs ? 1.6f : 1.0f);
  for (int i = 0; i < (glu ? kW4FewLinearOnly : (int)(sizeof(kW4Few) / sizeof(W4Shape))); ++i) {
    const W4Shape& s = kW4Few[i];
    // Beside two blocks of rows, and in sixteen waves, there are no registers for a g's halves; nor, beside the former,
    // for six columns' scales of small groups.
    if (gs && (s.rows == 32 || s.ks == 16)) continue;
    if (s.rows == 32 && (M <= 16 || (s.cols == 96 && group < 128))) continue;
    const int64_t wgs = (int64_t)((M + s.rows - 1) / s.rows) * ((NP + s.cols - 1) / s.cols);
    const float us = kW4FewUs + kW4FewPerMK * ((float)M * (float)K * 1e-6f) + x * shape_us(s, wgs, (KB + s.ks - 1) / s.ks);
    if (us < best.us) best = W4Best{{false, i, 1, KB}, us};
  }
  return best;
}

// Not looked for where no shape can take less than `bound`.
static W4Best many_plan(int M, int K, int KB, int NP, int group, float bound) {
  W4Best best{{true, 0, 1, KB}, 1e30f};
  const float fixed = kW4ManyUs + kW4ManyPerMK * ((float)M * (float)K * 1e-6f);
  if (fixed >= bound) return best;
  const float x = group == 32 ? 1.15f : group == 64 ? 1.04f : 1.0f;
  for (int i = 0; i < (int)(sizeof(kW4Many) / sizeof(W4Shape)); ++i) {
    const W4Shape& s = kW4Many[i];
    const int64_t tiles = (int64_t)((M + s.rows - 1) / s.rows) * ((NP + s.cols - 1) / s.cols);
    for (int splits = 1; splits <= 16; splits *= 2) {
      if (splits > 1 && (tiles * splits > 1100 || KB < 2 * splits)) break;
      const int per = ((KB + splits - 1) / splits + s.ks - 1) / s.ks * s.ks, n = (KB + per - 1) / per;
      float us = fixed + x * shape_us(s, tiles * n, per / s.ks);
      if (n > 1) us += kW4JoinUs + kW4JoinPerMB * (float)n * (float)M * (float)NP * 4e-6f;
      if (us < best.us) best = W4Best{{true, i, n, per}, us};
    }
  }
  return best;
}

W4Plan w4_plan(int M, int K, int KB, int NP, bool glu, int group, bool gs) {
  const W4Best few = few_plan(M, K, KB, NP, glu, group, gs);
  if (M <= FN_W4_FEW_M) return few.plan;
  const W4Best many = many_plan(M, K, KB, NP, group, few.us);
  return few.us <= many.us ? few.plan : many.plan;
}

// Rows that go through the kernels together: a launch has fewer than 2^32 threads, up to 1024 per workgroup and, in the
// many-row kernel's pass over the rows, up to 1024 per row.  0 where one block of rows is too many already.
static int64_t piece_rows(const W4Plan& plan, int64_t NP) {
  constexpr int64_t kMost = (int64_t(1) << 22) - 1;
  const W4Shape& s = plan.many ? kW4Many[plan.shape] : kW4Few[plan.shape];
  const int64_t rows = kMost / ((NP + s.cols - 1) / s.cols * plan.splits) * s.rows;
  return plan.many && rows > kMost ? kMost / s.rows * s.rows : rows;
}

// Workspace of a call: the rows' factors, the fp16 activations and the splits' sums; 0 for the few-row kernel.
static int64_t factor_bytes(int64_t M) { return round_up(M * 4, 256); }
int64_t w4_workspace(const W4Plan& plan, int64_t M, int64_t KB, int64_t NP) {
  if (!plan.many) return 0;
  const int64_t piece = piece_rows(plan, NP);
  if (M > piece) M = piece;
  return factor_bytes(M) + M * KB * (2 * kW4KB) + (plan.splits > 1 ? plan.splits * M * NP * 4 : 0);
}

int64_t w4_workspace(int64_t M, int64_t K, int64_t NP, bool glu, int group) {
  if (M <= FN_W4_FEW_M) return 0;
  const int KB = (int)w4_blocks(K);
  const float plain = few_plan((int)M, (int)K, KB, (int)NP, glu, group, false).us;
  const float with_g = few_plan((int)M, (int)K, KB, (int)NP, glu, group, true).us;
  const float slower = plain > with_g ? plain : with_g;
  const W4Best many = many_plan((int)M, (int)K, KB, (int)NP, group, slower);
  return slower <= many.us ? 0 : w4_workspace(many.plan, M, KB, NP);
}

template <bool NORM>
static hipError_t launch_w4_rows(const W4Args& p, _Float16* out, float* factor) {
  const int KP = p.KB * kW4KB;
  auto go = [&](auto kernel, int threads) {
    hipLaunchKernelGGL(kernel, dim3(p.M), dim3(threads), 0, p.stream, p.a, p.K, p.lda, p.ep.g_rt, p.ep.eps, p.ep.inv_k,
                       KP, out, factor, p.ep.inv_rms);
    return hipGetLastError();
  };
  // More threads for long rows where rows alone do not fill the chip (64 x 11008: the call 25.1 -> 22.5 us).
  if (KP <= 8192) return go(w4_rows_kernel<NORM, 256, 4>, 256);
  if (KP <= 32768) return go(w4_rows_kernel<NORM, 1024, 4>, 1024);
  return go(w4_rows_kernel<NORM, 1024, 0>, 1024);
}

static hipError_t launch_w4_piece(const W4Args& p) {
  const W4Plan& plan = p.plan;
  if (!plan.many) {
    switch (p.epi) {
      case EPI_RMS: return launch_w4_few<EPI_RMS>(p, plan.shape);
      case EPI_GLU: return launch_w4_few<EPI_GLU>(p, plan.shape);
      case EPI_ROWSCALE: return launch_w4_few<EPI_ROWSCALE>(p, plan.shape);
    }
    return hipErrorInvalidValue;
  }
  char* ws = static_cast<char*>(p.ws);
  float* factor = reinterpret_cast<float*>(ws);
  _Float16* act = reinterpret_cast<_Float16*>(ws + factor_bytes(p.M));
  float* partial = reinterpret_cast<float*>(ws + factor_bytes(p.M) + (int64_t)p.M * p.KB * (2 * kW4KB));
  const hipError_t e = p.epi == EPI_ROWSCALE ? launch_w4_rows<false>(p, act, factor) : launch_w4_rows<true>(p, act, factor);
  if (e != hipSuccess) return e;
  const int rows = kW4Many[plan.shape].rows, groups = (p.M + rows - 1) / rows;
  // Row groups that share a column tile's codes in an XCD's L2: all of them where their activations fit it (4 MB)
  // beside each other, else pairs, whose activations it holds while the tiles go by.  All / pairs: 333 x 4096 -> 12288
  // 58.2 / 61.0 us, 2048 x 11008 -> 4096 187 / 177; panels of four and eight are no better there.
  const int panel = (int64_t)p.M * p.KB * (2 * kW4KB) <= (4 << 20) ? groups : 2;
  const W4Gemm q{act, p.M, p.KB * kW4KB, p.codes, p.scales, p.norms, p.NP, p.KB, p.ncols, factor, p.ep.row_scale,
                 p.ep.bias, p.y, p.ldy, groups, panel, plan.splits, plan.kb_per_split, partial};
  switch (p.epi) {
    case EPI_RMS: return launch_w4_many<EPI_RMS>(q, p.group, plan.shape, p.stream);
    case EPI_GLU: return launch_w4_many<EPI_GLU>(q, p.group, plan.shape, p.stream);
    case EPI_ROWSCALE: return launch_w4_many<EPI_ROWSCALE>(q, p.group, plan.shape, p.stream);
  }
  return hipErrorInvalidValue;
}

// More rows than a launch takes go in pieces, one after the other on the stream and in the same workspace.
hipError_t launch_w4(const W4Args& p) {
  constexpr int64_t kPieces = 1024;  // beyond, the output has some 2^40 elements
  const int64_t piece = piece_rows(p.plan, p.NP);
  if (p.M <= piece) return launch_w4_piece(p);
  if (p.M > piece * kPieces) return hipErrorInvalidConfiguration;
  for (int64_t m = 0; m < p.M; m += piece) {
    W4Args q = p;
    q.M = (int)(p.M - m < piece ? p.M - m : piece);
    q.a += m * p.lda;
    q.y += m * p.ldy;
    if (q.ep.inv_rms) q.ep.inv_rms += m;
    if (q.ep.row_scale) q.ep.row_scale += m;
    const hipError_t e = launch_w4_piece(q);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace fn
