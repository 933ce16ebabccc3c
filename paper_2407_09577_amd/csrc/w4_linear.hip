// Products with 4-bit weights: RMSNorm -> linear / GLU and the row-scaled linear layer, deferred as in
// the bf16 kernels, with the codes of fn_w4.h.
#include "fn_device.h"
#include "fn_epilogue.h"
#include "fn_launch.h"
#include "fn_w4.h"

namespace fn {

// A workgroup owns 16 rows and NCB column blocks; its KS waves take the 128-row code blocks in turn and
// their partial products meet in LDS in a fixed order.
template <int NCB, int KS, int GB, int EPI>
__global__ __launch_bounds__(64 * KS) void w4_rows_kernel(const __bf16* __restrict__ a, int M, int K, int lda,
                                                          const void* __restrict__ codes,
                                                          const unsigned* __restrict__ scales, int NP, int KB,
                                                          int ncols, __bf16* __restrict__ y, int ldy, EpiArgs ep,
                                                          int tiles) {
  constexpr bool kSS = epi_needs_ss(EPI);
  constexpr int NG = 4 / GB;
  __shared__ f32x4 red[KS][NCB][64];
  __shared__ float red_ss[KS][16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile = blockIdx.x % tiles, cb0 = tile * NCB, npb = NP / 16;
  const int m0 = blockIdx.x / tiles * 16, rows = min(16, M - m0);
  const int lrow = lane & 15, lch = lane >> 4;
  const __amdgpu_buffer_rsrc_t rs_a =
      make_rsrc(a + (int64_t)m0 * lda, (uint32_t)(((int64_t)(rows - 1) * lda + K) * 2));
  // Column blocks past the packed width (last workgroup only) read other codes, or zeros past the end;
  // their outputs are never stored.
  const __amdgpu_buffer_rsrc_t rs_w = make_rsrc(codes, (uint32_t)((int64_t)KB * npb * 1024));
  const __amdgpu_buffer_rsrc_t rs_s = make_rsrc(scales, (uint32_t)((int64_t)KB * NG * NP * 4));
  const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});

  f32x4 acc[NCB];
#pragma unroll
  for (int c = 0; c < NCB; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  float ss = 0.f;
  for (int kb = wave; kb < KB; kb += KS) {
    u32x4 wf[NCB], sf[NG][NCB], af[4];
#pragma unroll
    for (int c = 0; c < NCB; ++c)
      wf[c] = load_buf16<kCachePolicyNT>(rs_w, (unsigned)(kb * npb + cb0 + c) * 1024u + lane * 16);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int k = kb * kW4KB + 32 * u + 8 * lch;
      af[u] = load_buf16(rs_a, lrow < rows && k < K ? (unsigned)(lrow * lda + k) * 2 : kOobOffset);
    }
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int c = 0; c < NCB; ++c)
        sf[j][c] = load_buf16(rs_s, (unsigned)((kb * NG + j) * NP + (cb0 + c) * 16 + lch * 4) * 4u);
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      f32x4 part[NCB], sum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NCB; ++c) part[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = j * GB; u < (j + 1) * GB; ++u) {
        bf16x8 av = __builtin_bit_cast(bf16x8, af[u]);
        if constexpr (kSS) ss = sumsq8(av, ss);
        bf16x8 lo = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
        if (ep.g_rt) {  // a g as two bf16: its rounding and what that leaves
          const int k = kb * kW4KB + 32 * u + 8 * lch;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float o = k < K ? (float)av[e] * ep.g_rt[k + e] : 0.0f;
            av[e] = (__bf16)o;
            lo[e] = (__bf16)(o - (float)av[e]);
          }
          sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, lo, sum, 0, 0, 0);
#pragma unroll
          for (int c = 0; c < NCB; ++c)
            part[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w4_widen(wf[c][u]), lo, part[c], 0, 0, 0);
        }
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, av, sum, 0, 0, 0);
#pragma unroll
        for (int c = 0; c < NCB; ++c)
          part[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w4_widen(wf[c][u]), av, part[c], 0, 0, 0);
      }
#pragma unroll
      for (int c = 0; c < NCB; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const unsigned sw = sf[j][c][r];
          acc[c][r] = fmaf(w4_scale(sw), fmaf(-((float)kW4Bias + w4_zero(sw)), sum[0], part[c][r]), acc[c][r]);
        }
    }
  }
  if constexpr (kSS) {
    ss += __shfl_xor(ss, 16);
    ss += __shfl_xor(ss, 32);
  }
#pragma unroll
  for (int c = 0; c < NCB; ++c) red[wave][c][lane] = acc[c];
  if (lane < 16) red_ss[wave][lane] = ss;
  __syncthreads();
  const int m = m0 + lrow;
  if (m >= M) return;
  float ss_t = 0.f;
#pragma unroll
  for (int w = 0; w < KS; ++w) ss_t += red_ss[w][lrow];
  RowStat st = row_stat<EPI>(ss_t, 0.f, ep);
  if constexpr (EPI == EPI_ROWSCALE) st.s = ep.row_scale ? ep.row_scale[m] : 1.0f;
  if constexpr (epi_exports_s(EPI)) {
    if (ep.inv_rms && tile == 0 && wave == 0 && lane < 16) ep.inv_rms[m] = st.s;
  }
  auto total = [&](int c) __attribute__((always_inline)) {
    f32x4 v = red[0][c][lane];
#pragma unroll
    for (int w = 1; w < KS; ++w) v += red[w][c][lane];
    return v;
  };
  constexpr int STEP = epi_is_glu(EPI) ? 2 : 1;
  for (int o = wave; o < NCB / STEP; o += KS) {
    const f32x4 v = total(o * STEP), u = STEP == 2 ? total(o * STEP + 1) : v;
    const int n = (cb0 / STEP + o) * 16 + lch * 4;
    if (epi_vec<EPI>(ep)) {
      if (n + 4 <= ncols) store4_bf16_full<EPI, true>(y, ldy, m, n, v, u, st, ep);
      else store4_bf16_edge<EPI, true>(y, ldy, M, ncols, m, n, v, u, st, ep);
    } else {
      if (n + 4 <= ncols) store4_bf16_full<EPI, false>(y, ldy, m, n, v, u, st, ep);
      else store4_bf16_edge<EPI, false>(y, ldy, M, ncols, m, n, v, u, st, ep);
    }
  }
}

template <int GB, int EPI>
static hipError_t launch_w4_t(const W4Args& p) {
  constexpr int NCB = 2, KS = 4;
  const int tiles = (p.NP / 16 + NCB - 1) / NCB;
  const int64_t blocks = (int64_t)tiles * ((p.M + 15) / 16);
  if (blocks * 64 * KS >= (int64_t(1) << 32)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((w4_rows_kernel<NCB, KS, GB, EPI>), dim3((unsigned)blocks), dim3(64 * KS), 0, p.stream, p.a, p.M, p.K, p.lda, p.codes,
                     p.scales, p.NP, p.KB, p.ncols, p.y, p.ldy, p.ep, tiles);
  return hipGetLastError();
}

template <int EPI>
static hipError_t launch_w4_epi(const W4Args& p) {
  return p.group == 32 ? launch_w4_t<1, EPI>(p) : p.group == 64 ? launch_w4_t<2, EPI>(p) : launch_w4_t<4, EPI>(p);
}

hipError_t launch_w4(const W4Args& p) {
  switch (p.epi) {
    case EPI_RMS: return launch_w4_epi<EPI_RMS>(p);
    case EPI_GLU: return launch_w4_epi<EPI_GLU>(p);
    case EPI_ROWSCALE: return launch_w4_epi<EPI_ROWSCALE>(p);
  }
  return hipErrorInvalidValue;
}

}  // namespace fn
