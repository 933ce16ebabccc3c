// Kernels of the products with 4-bit weights (layout and arithmetic: fn_w4.h).
#pragma once

#include <type_traits>

#include "fn_device.h"
#include "fn_epilogue.h"
#include "fn_launch.h"
#include "fn_tile.h"
#include "fn_w4.h"

namespace fn {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

// One output from its accumulator (GLU: gate and up), the row's scale and the column's bias.
template <int EPI>
__device__ __forceinline__ float w4_value(float v, float u, float s, float bias) {
  return epi_value<EPI>(v, u, RowStat{s, 0.0f, 0}, bias, 0.0f);
}

template <int EPI>
__device__ __forceinline__ float w4_row_scale(float ss, const EpiArgs& ep, int m) {
  if constexpr (EPI == EPI_ROWSCALE) return ep.row_scale ? ep.row_scale[m] : 1.0f;
  else return row_stat<EPI>(ss, 0.0f, ep).s;
}

// a g as two bf16, its rounding and what that leaves (2^-17 of it): one bf16 alone would add an error
// as large as the output's own rounding.
__device__ __forceinline__ void split_ag(const bf16x8& a, const f32x4& g0, const f32x4& g1, bf16x8& hi, bf16x8& lo) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float o = (float)a[e] * (e < 4 ? g0[e & 3] : g1[e & 3]);
    hi[e] = (__bf16)o;
    lo[e] = (__bf16)(o - (float)hi[e]);
  }
}

// Few rows: bound by the weight stream.  A workgroup owns RG blocks of 16 rows and NCB column blocks; its KS waves
// take code blocks (128 k each) in turn, the next one's loads in flight while the present one is multiplied, and
// the partial products meet in LDS in a fixed order.
// A wave's activations come straight in the matrix-core order, where sixteen rows lie in one load, or STAGED: read
// along the rows and turned in a slot of LDS of its own.  That halves the requests of a load of sixteen rows
// (4096 -> 6144 with one column block a wave: 11.9 -> 9.1 us) and only adds a wait to one of a row or two
// (two blocks: 6.6 -> 7.6).
// Kernel times: 1 x 4096 -> 6144 6.8 us, 16 x 4096 -> 22016 GLU 13.8 us for 50 MB, beside 3.1 us of a kernel that does
// nothing: the stream itself runs at 3.7 to 4.7 TB/s.  64 x 11008 -> 4096 (17.7 us a call, 20 to 22 traced one by one)
// widens every code once for each 16 rows and waits in between: vector instructions issue for a third of the time, the
// matrix cores are busy for an eighth.  Loads two blocks ahead gained 5% at K = 11008 and cost as much at 4096.
template <int NCB, int KS, int RG, int GB, int EPI, bool GS, bool STAGED>
__global__ __launch_bounds__(64 * KS) void w4_few_kernel(const __bf16* __restrict__ a, int M, int K, int lda,
                                                         const void* __restrict__ codes,
                                                         const unsigned* __restrict__ scales, int NP, int KB, int ncols,
                                                         __bf16* __restrict__ y, int ldy, EpiArgs ep, int groups) {
  constexpr bool kSS = epi_needs_ss(EPI);
  constexpr int NG = 4 / GB, STEP = epi_is_glu(EPI) ? 2 : 1;
  static_assert(NCB % STEP == 0, "GLU needs gate/up block pairs");
  // Each wave's slot for a block's activations, then (behind a barrier) the partial products.
  static_assert(STAGED || (!GS && RG == 1), "a g is split on its way through LDS, and 32 rows are turned there");
  constexpr int PLANES = GS ? 2 : 1, SLOT = STAGED ? 256 * PLANES * RG : 0;  // units of a wave's slot
  constexpr int UNITS = KS * (SLOT > 64 * NCB * RG ? SLOT : 64 * NCB * RG);
  __shared__ u32x4 smem[UNITS];
  __shared__ float red_ss[KS][16 * RG];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // The row groups of a column tile are neighbours on one XCD and share its codes in that L2.
  const int q8 = gridDim.x / kXcds, r8 = gridDim.x % kXcds, x8 = blockIdx.x % kXcds;
  const int logical = x8 * q8 + min(x8, r8) + blockIdx.x / kXcds;
  const int tile = logical / groups, m0 = logical % groups * (16 * RG), rows = min(16 * RG, M - m0);
  const int cb0 = tile * NCB, npb = NP / 16;
  const int lrow = lane & 15, lch = lane >> 4;
  const __amdgpu_buffer_rsrc_t rs_a =
      make_rsrc(a + (int64_t)m0 * lda, (uint32_t)(((int64_t)(rows - 1) * lda + K) * 2));
  const __amdgpu_buffer_rsrc_t rs_g = make_rsrc(ep.g_rt, GS ? (uint32_t)K * 4u : 0u);
  // Column blocks past the packed width (last workgroup only) read other codes, or zeros past the end;
  // their outputs are never stored.
  const __amdgpu_buffer_rsrc_t rs_w = make_rsrc(codes, (uint32_t)((int64_t)KB * npb * 1024));
  const __amdgpu_buffer_rsrc_t rs_s = make_rsrc(scales, (uint32_t)((int64_t)KB * NG * NP * 4));
  const unsigned one2 = 0x3f803f80u;  // bf16 1, twice
  const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{one2, one2, one2, one2});

  const W4Bits bits(0x43004300u);

  struct Set {
    u32x4 w[NCB], a[RG][4], g[GS ? 2 : 1];
    unsigned s[NG][NCB];
  };
  auto load_set = [&](int kb, Set& t) __attribute__((always_inline)) {
    const bool ok = kb < KB;
#pragma unroll
    for (int c = 0; c < NCB; ++c)
      t.w[c] = load_buf16<kCachePolicyNT>(rs_w, ok ? (unsigned)(kb * npb + cb0 + c) * 1024u + lane * 16 : kOobOffset);
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int c = 0; c < NCB; ++c)
        t.s[j][c] = __builtin_amdgcn_raw_buffer_load_b32(
            rs_s, ok ? (unsigned)((kb * NG + j) * NP + (cb0 + c) * 16 + lrow) * 4u : kOobOffset, 0, 0);
#pragma unroll
    for (int q = 0; q < RG; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // Staged: sixteen lanes read one row's 256 bytes, four rows at a time.  Else: the matrix-core order.
        const int row = 16 * q + (STAGED ? 4 * j + lch : lrow), k = kb * kW4KB + (STAGED ? 8 * lrow : 32 * j + 8 * lch);
        if (GS && 4 * j >= rows) continue;  // what a row costs is its splitting (else the branch costs more)
        t.a[q][j] = load_buf16(rs_a, row < rows && k < K ? (unsigned)(row * lda + k) * 2 : kOobOffset);
      }
    if constexpr (GS) {  // this lane's eight k, the same for its four rows; past K: zeros
      const unsigned k = (unsigned)(kb * kW4KB + 8 * lrow);
      t.g[0] = load_buf16(rs_g, k * 4);
      t.g[1] = load_buf16(rs_g, k * 4 + 16);
    }
  };
  // Piece (k block u, chunk c) of row r in the slot: where the matrix-core order reads it, at a position XORed
  // so that the sixteen pieces of a row are written to different banks.
  auto slot = [](int u, int r, int c) { return u * 64 + 16 * c + (r ^ (c + 4 * u)); };
  u32x4* own = smem + wave * SLOT;
  if constexpr (GS) {
    if (rows <= 12) {
#pragma unroll
      for (int i = 0; i < SLOT / 64; ++i) own[i * 64 + lane] = u32x4{0, 0, 0, 0};
    }
  }
  f32x4 acc[RG][NCB];
  float ss[RG], ss4[4] = {0.f, 0.f, 0.f, 0.f};  // ss4, with g: of the raw rows 4 j + lch
#pragma unroll
  for (int q = 0; q < RG; ++q) {
    ss[q] = 0.f;
#pragma unroll
    for (int c = 0; c < NCB; ++c) acc[q][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto compute_set = [&](const Set& t) __attribute__((always_inline)) {
    if constexpr (STAGED) {
      wave_lds_order();
#pragma unroll
      for (int q = 0; q < RG; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (GS && 4 * j >= rows) continue;  // the slot holds zeros there
          const int at = slot(lrow >> 2, 4 * j + lch, lrow & 3);
          if constexpr (GS) {
            bf16x8 hi, lo;
            if constexpr (kSS) ss4[j] = sumsq8(__builtin_bit_cast(bf16x8, t.a[q][j]), ss4[j]);
            split_ag(__builtin_bit_cast(bf16x8, t.a[q][j]), __builtin_bit_cast(f32x4, t.g[0]),
                     __builtin_bit_cast(f32x4, t.g[1]), hi, lo);
            own[at] = __builtin_bit_cast(u32x4, hi);
            own[256 + at] = __builtin_bit_cast(u32x4, lo);
          } else {
            own[256 * q + at] = t.a[q][j];
          }
        }
      wave_lds_order();
    }
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      bf16x8 av[RG][GB], al[GB];
      f32x4 sum[RG];  // the group's sum of each row's activations
#pragma unroll
      for (int q = 0; q < RG; ++q) {
        sum[q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < GB; ++b) {
          const int u = j * GB + b;
          av[q][b] = __builtin_bit_cast(bf16x8, STAGED ? own[256 * q + slot(u, lrow, lch)] : t.a[q][u]);
          if constexpr (kSS && !GS) ss[q] = sumsq8(av[q][b], ss[q]);
          if constexpr (GS) {
            al[b] = __builtin_bit_cast(bf16x8, own[256 + slot(u, lrow, lch)]);
            sum[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(al[b], ones, sum[q], 0, 0, 0);
          }
          sum[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[q][b], ones, sum[q], 0, 0, 0);
        }
      }
#pragma unroll
      for (int c = 0; c < NCB; ++c) {
        f32x4 part[RG];
#pragma unroll
        for (int q = 0; q < RG; ++q) part[q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < GB; ++b) {
          const bf16x8 wv = w4_widen(t.w[c][j * GB + b], bits);
          if constexpr (GS) part[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(al[b], wv, part[0], 0, 0, 0);
#pragma unroll
          for (int q = 0; q < RG; ++q) part[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[q][b], wv, part[q], 0, 0, 0);
        }
        const float s = w4_scale(t.s[j][c]), bias = -kW4Bias - w4_zero(t.s[j][c]);
#pragma unroll
        for (int q = 0; q < RG; ++q)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[q][c][r] = fmaf(s, fmaf(bias, sum[q][r], part[q][r]), acc[q][c][r]);
      }
    }
  };
  Set t0, t1;
  load_set(wave, t0);
  for (int kb = wave; kb < KB; kb += 2 * KS) {
    load_set(kb + KS, t1);
    __builtin_amdgcn_sched_barrier(0);
    compute_set(t0);
    __builtin_amdgcn_sched_barrier(0);
    if (kb + KS >= KB) break;
    load_set(kb + 2 * KS, t0);
    __builtin_amdgcn_sched_barrier(0);
    compute_set(t1);
    __builtin_amdgcn_sched_barrier(0);
  }

  if constexpr (kSS && GS) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) ss4[j] += __shfl_xor(ss4[j], o);
      if (lrow == 0) red_ss[wave][4 * j + lch] = ss4[j];
    }
  } else if constexpr (kSS) {
#pragma unroll
    for (int q = 0; q < RG; ++q) {
      ss[q] += __shfl_xor(ss[q], 16);
      ss[q] += __shfl_xor(ss[q], 32);
      if (lane < 16) red_ss[wave][16 * q + lane] = ss[q];
    }
  }
  __syncthreads();
  f32x4* red = reinterpret_cast<f32x4*>(smem);
#pragma unroll
  for (int q = 0; q < RG; ++q)
#pragma unroll
    for (int c = 0; c < NCB; ++c) red[((wave * RG + q) * NCB + c) * 64 + lane] = acc[q][c];
  __syncthreads();
  constexpr int OUTS = NCB / STEP;  // output column blocks
  for (int i = wave; i < RG * OUTS; i += KS) {
    const int q = i / OUTS, o = i % OUTS;
    f32x4 v = {0.f, 0.f, 0.f, 0.f}, u = v;
#pragma unroll
    for (int w = 0; w < KS; ++w) {
      v += red[((w * RG + q) * NCB + o * STEP) * 64 + lane];
      if constexpr (STEP == 2) u += red[((w * RG + q) * NCB + o * STEP + 1) * 64 + lane];
    }
    const int n = (cb0 / STEP + o) * 16 + lrow;
    const float bias = EPI == EPI_RMS && ep.bias && n < ncols ? ep.bias[n] : 0.0f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * q + 4 * lch + r, m = m0 + row;
      if (row >= rows) break;
      float ss_t = 0.f;
      if constexpr (kSS) {
#pragma unroll
        for (int w = 0; w < KS; ++w) ss_t += red_ss[w][row];
      }
      const float s = w4_row_scale<EPI>(ss_t, ep, m);
      if constexpr (epi_exports_s(EPI)) {
        if (ep.inv_rms && tile == 0 && o == 0 && lrow == 0) ep.inv_rms[m] = s;
      }
      if (n < ncols) y[(int64_t)m * ldy + n] = (__bf16)w4_value<EPI>(v[r], u[r], s, bias);
    }
  }
}

// Many rows: the activations are brought to fp16 first (w4_rows_kernel), each row times the power of two
// that puts its largest value into [2^14, 2^15), and a weight is widened to the fp16 of (q - z) r, r its
// group's scale times a power of two of the column.  Eleven bits hold a bf16 activation exactly and round
// a weight by 2^-12 at most, an eighth of the output's own rounding in the sums' root mean square, and what
// lies 2^-29 below a row's largest value or 2^-24 below a column's largest scale fades into the subnormals: their
// steps of 2^-24 leave an activation off by at most 2^-39 of the row's largest value, and a weight by (|q - z| + 1) 2^-25
// of the column's power of two, 2^-28 of its largest scale.
// So the matrix cores sum over all of K: no group of k needs a sum of its own, and no activation statistics
// are left to the product.
//
// One workgroup per row: the row's squares and largest value, then its fp16 form, [KB * 128] with zeros
// past K, and the factor that the outputs take: 1 / the power of two, and 1 / RMSe times that.  A given row scale
// comes after it: the product of the two could leave fp32 where neither does.
// With g the values are a g, rounded to fp16, 2^-12 of each at most: an error in the outputs of a twelfth of their own
// rounding (root mean square), where the few-row kernel's two halves would double the products.
// A row that holds a NaN or an infinity gets a NaN factor.
// T threads hold up to H pieces of 16 bytes each; H = 0: the row is read twice.  Bound by its launch and one trip to
// memory: 333 x 4096 5.2 us, 2048 x 4096 10.5 us.
template <bool NORM, int T, int H>
__global__ __launch_bounds__(T) void w4_rows_kernel(const __bf16* __restrict__ a, int K, int lda,
                                                    const float* __restrict__ g, float eps, float inv_k, int KP,
                                                    _Float16* __restrict__ out, float* __restrict__ factor,
                                                    float* __restrict__ inv_rms) {
  __shared__ float red[T / 64];
  __shared__ unsigned red_top[T / 64];
  const int64_t m = blockIdx.x;
  const __bf16* ar = a + m * lda;
  float ss = 0.f;
  unsigned top = 0;  // bits of the largest magnitude: floats without a sign are ordered as their bits are
  auto widen = [&](const u32x4& w, int k, float (&v)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bf16_lo(w[i]), v[2 * i + 1] = bf16_hi(w[i]);
    if (g) {
      const f32x4 g0 = *reinterpret_cast<const f32x4*>(g + k), g1 = *reinterpret_cast<const f32x4*>(g + k + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= g0[e], v[4 + e] *= g1[e];
    }
  };
  auto measure = [&](const u32x4& w, int k) __attribute__((always_inline)) {
    if constexpr (NORM) ss = sumsq8(__builtin_bit_cast(bf16x8, w), ss);
    float v[8];
    widen(w, k, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
  };
  auto put = [&](const u32x4& w, int k, float f) __attribute__((always_inline)) {
    f16x8 h = {0, 0, 0, 0, 0, 0, 0, 0};
    if (k < K) {
      float v[8];
      widen(w, k, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = (_Float16)(v[e] * f);
    }
    *reinterpret_cast<f16x8*>(out + m * KP + k) = h;
  };
  u32x4 held[H ? H : 1];
  if constexpr (H > 0) {
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const int k = (i * T + threadIdx.x) * 8;
      held[i] = u32x4{0, 0, 0, 0};
      if (k < K) held[i] = *reinterpret_cast<const u32x4*>(ar + k);
    }
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const int k = (i * T + threadIdx.x) * 8;
      if (k < K) measure(held[i], k);
    }
  } else {
    for (int k = threadIdx.x * 8; k < K; k += T * 8) measure(*reinterpret_cast<const u32x4*>(ar + k), k);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    if constexpr (NORM) ss += __shfl_xor(ss, o);
    top = max(top, (unsigned)__shfl_xor((int)top, o));
  }
  if ((threadIdx.x & 63) == 0) {
    red[threadIdx.x >> 6] = ss;
    red_top[threadIdx.x >> 6] = top;
  }
  __syncthreads();
  ss = red[0];
  top = red_top[0];
#pragma unroll
  for (int w = 1; w < T / 64; ++w) {
    ss += red[w];
    top = max(top, red_top[w]);
  }
  const unsigned ex = top >> 23;
  const float f = ex == 255u ? 1.0f : __uint_as_float(min(268u - ex, 254u) << 23);
  if (threadIdx.x == 0) {
    float s = 1.0f;
    if constexpr (NORM) {
      s = rsqrtf(fmaf(ss, inv_k, eps));
      if (inv_rms) inv_rms[m] = s;
    }
    factor[m] = ex == 255u ? __builtin_nanf("") : s * (1.0f / f);
  }
  if constexpr (H > 0) {
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const int k = (i * T + threadIdx.x) * 8;
      if (k < KP) put(held[i], k, f);
    }
  } else {
    for (int k = threadIdx.x * 8; k < KP; k += T * 8) {
      const u32x4 w = k < K ? *reinterpret_cast<const u32x4*>(ar + k) : u32x4{0, 0, 0, 0};
      put(w, k, f);
    }
  }
}

// The eight weights of a word as fp16 (q - z) r, in k order.  zero holds 1024 + z twice, zero64 64 + z, r the group's
// scale.  The odd nibbles are taken where they stand, 1024 + 16 q, whose sixteenth less 64 + z is q - z again, exactly:
// a sixteenth of r instead would be subnormal, and lose bits, sixteen times sooner than r.
__device__ __forceinline__ f16x8 w4_widen_f16(unsigned w, const W4Bits& k, f16x2 zero, f16x2 zero64, f16x2 r) {
  auto at = [](unsigned v) { return __builtin_bit_cast(f16x2, v); };
  const f16x2 sixteenth = {0.0625, 0.0625};
  const unsigned h = w >> 8;
  const f16x2 p0 = (at((w & k.low) | k.bias) - zero) * r;
  const f16x2 p1 = __builtin_elementwise_fma(at((w & k.high) | k.bias), sixteenth, -zero64) * r;
  const f16x2 p2 = (at((h & k.low) | k.bias) - zero) * r;
  const f16x2 p3 = __builtin_elementwise_fma(at((h & k.high) | k.bias), sixteenth, -zero64) * r;
  return f16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// A workgroup owns 16 MB WM rows and 16 NCB WN packed columns; its waves are WM row waves, WN column waves
// and KS k groups, and a set is KS code blocks (128 k each).  Codes and scale words go from memory straight
// into the registers of the waves that multiply them, one set ahead.  The activations go by LDS-DMA into a
// ring of NST stages, NST - 1 sets ahead: 16 lanes bring one row's 256 bytes, 16-byte piece j of row r at
// position j ^ (r % 16), so that the sixteen rows of an operand read lie in different banks.
// With several `splits` of K each workgroup writes its fp32 sums and w4_join_kernel finishes them.
// 2048 x 4096 -> 22016 GLU takes 316 to 337 us on different cards, 1.10 to 1.17 PFLOP/s: the matrix cores are busy for
// half of the time, and the vector instructions that widen issue for a third.  With fewer workgroups it is the waits in
// one set that count: a set of 128 k takes a workgroup that is alone on its compute unit 2600 cycles, 1024 of them
// matrix-core operations.  Weights through LDS as well, a third stage,
// operands read six or eight steps ahead and widening spread over the steps, into the next set's first, did not help.
struct W4Gemm {
  const _Float16* a;  // [M][KP]
  int M, KP;
  const void* codes;
  const unsigned* scales;
  const float* col_norm;  // [NP] the columns' powers of two
  int NP, KB, ncols;
  const float* factor;     // [M]
  const float* row_scale;  // EPI_ROWSCALE: optional [M]
  const float* bias;
  __bf16* y;
  int ldy;
  int groups, panel;  // row groups, and how many of them go through the column tiles together
  int splits, kb_per_split;
  float* partial;  // [splits][M][NP]
};

// One output of the many-row kernel from its sums, the row's factor and the columns' 1 / norm.
template <int EPI>
__device__ __forceinline__ float w4_many_value(float v, float u, float n0, float n1, float factor, float scale, float bias) {
  if constexpr (EPI == EPI_ROWSCALE) return v * n0 * factor * scale;
  else return w4_value<EPI>(v * n0, u * n1, factor, bias);
}

template <int EPI>
__device__ __forceinline__ float w4_given_scale(const W4Gemm& p, int64_t m) {
  return EPI == EPI_ROWSCALE && p.row_scale ? p.row_scale[m] : 1.0f;
}

template <int MB, int NCB, int WM, int WN, int KS, int NST, int GB, int EPI>
__global__ __launch_bounds__(64 * WM * WN * KS, 2) void w4_gemm_kernel(W4Gemm p) {
  constexpr int NW = WM * WN * KS, NG = 4 / GB, STEP = epi_is_glu(EPI) ? 2 : 1;
  constexpr int ROWS = 16 * MB * WM, CB = WN * NCB;
  constexpr int STAGE = ROWS * 256 * KS;    // bytes
  constexpr int ND = ROWS * KS / (4 * NW);  // transfers of 1 KiB (4 rows) per wave and set
  static_assert(ROWS * KS % (4 * NW) == 0 && NCB % STEP == 0, "whole transfers; gate/up pairs");
  constexpr int OUTC = CB * 16 / STEP, PITCH = OUTC + 8;
  constexpr int RING = NST * STAGE, RED = (KS - 1) * WM * MB * CB * 1024, OUT = ROWS * PITCH * 2;
  constexpr int SMEM = RING > RED ? (RING > OUT ? RING : OUT) : (RED > OUT ? RED : OUT);
  __shared__ __align__(1024) char smem[SMEM];

  const int q8 = gridDim.x / kXcds, r8 = gridDim.x % kXcds, x8 = blockIdx.x % kXcds;
  int logical = x8 * q8 + min(x8, r8) + blockIdx.x / kXcds;
  const int tiles = (p.NP / 16 + CB - 1) / CB, panel = logical / (p.panel * tiles * p.splits);
  logical -= panel * (p.panel * tiles * p.splits);
  const int in_panel = min(p.panel, p.groups - panel * p.panel), grp = panel * p.panel + logical % in_panel;
  logical /= in_panel;
  const int split = logical % p.splits, tile = logical / p.splits;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = wave % WN, wm = wave / WN % WM, kg = wave / (WN * WM);
  const int cb0 = (tile * WN + wn) * NCB, npb = p.NP / 16;
  const int m0 = grp * ROWS, rows = min(ROWS, p.M - m0);
  const int lrow = lane & 15, lch = lane >> 4;
  const int kb_begin = split * p.kb_per_split, kb_end = min(p.KB, kb_begin + p.kb_per_split);
  const i32x4 rs_a = make_rsrc_sgpr(p.a + (int64_t)m0 * p.KP, (uint32_t)((int64_t)rows * p.KP * 2));
  const __amdgpu_buffer_rsrc_t rs_w = make_rsrc(p.codes, (uint32_t)((int64_t)p.KB * npb * 1024));
  const __amdgpu_buffer_rsrc_t rs_s = make_rsrc(p.scales, (uint32_t)((int64_t)p.KB * NG * p.NP * 4));

  // Transfer i of a wave: rows (i NW + wave) 4 .. + 3 of the set's KS x ROWS rows of 256 bytes.  Rows past M
  // and blocks past the split's end bring zeros: their offsets lie beyond the extent, which is below 2^30.
  constexpr unsigned kPast = 0x60000000u;
  static_assert(ROWS % (4 * NW) == 0, "a wave's rows are 4 NW apart, in one k group after the other");
  const unsigned a_off = (unsigned)((wave * 4 + lch) * p.KP) * 2u + (unsigned)((lrow ^ ((wave * 4 + lch) & 15)) * 16);
  auto load_act = [&](int kb0, int st) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      const int row4 = (i * NW + wave) * 4, j = i * NW * 4 / ROWS;
      const unsigned at = (unsigned)(i * NW * 4 % ROWS * p.KP + (kb0 + j) * kW4KB) * 2u;
      load_lds16(rs_a, smem + st * STAGE + row4 * 256, a_off + (kb0 + j < kb_end ? at : kPast));
    }
  };
  struct Weights {
    u32x4 w[NCB];
    unsigned s[NG][NCB];
  };
  // Past the split's end any block does, as its activations are zeros: the last one.  Column blocks past the
  // packed width (last tile only) read other codes, or zeros past the end; their outputs are never stored.
  const unsigned w_off = (unsigned)cb0 * 1024u + lane * 16, s_off = (unsigned)(cb0 * 16 + lrow) * 4u;
  auto load_w = [&](int kb0, Weights& t) __attribute__((always_inline)) {
    const int kb = min(kb0 + kg, p.KB - 1);
    const unsigned wk = w_off + (unsigned)(kb * npb) * 1024u;
#pragma unroll
    for (int c = 0; c < NCB; ++c) t.w[c] = load_buf16(rs_w, wk + c * 1024u);
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      const unsigned sk = s_off + (unsigned)((kb * NG + j) * p.NP) * 4u;
#pragma unroll
      for (int c = 0; c < NCB; ++c) t.s[j][c] = __builtin_amdgcn_raw_buffer_load_b32(rs_s, sk + c * 64u, 0, 0);
    }
  };
  float norm[NCB];
#pragma unroll
  for (int c = 0; c < NCB; ++c) norm[c] = cb0 + c < npb ? p.col_norm[(cb0 + c) * 16 + lrow] : 1.0f;
  f32x4 acc[MB][NCB];
#pragma unroll
  for (int t = 0; t < MB; ++t)
#pragma unroll
    for (int c = 0; c < NCB; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int rbase = (kg * ROWS + wm * MB * 16 + lrow) * 256;
  const W4Bits bits(0x64006400u);
  auto compute = [&](int st, const Weights& t) __attribute__((always_inline)) {
    const char* stage = smem + st * STAGE + rbase;
    auto zero_of = [&](int j, int c) __attribute__((always_inline)) {
      const unsigned z = t.s[j][c] & 63u;
      return __builtin_bit_cast(f16x2, 0x64006400u + (z | z << 16));
    };
    auto scale_of = [&](int j, int c) __attribute__((always_inline)) {
      const _Float16 h = (_Float16)(w4_scale(t.s[j][c]) * norm[c]);
      return f16x2{h, h};
    };
    // Kept over the k blocks that share them; with a group per k block they are made where they are used
    // (held ahead they cost 32 registers, and the 128 x 256 shape spilled its sums).
    f16x2 zero[NG < 4 ? NG : 1][NCB], r[NG < 4 ? NG : 1][NCB];
    if constexpr (NG < 4) {
#pragma unroll
      for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int c = 0; c < NCB; ++c) zero[j][c] = zero_of(j, c), r[j][c] = scale_of(j, c);
    }
    // Steps of one row block of one k block of 32: its operand is read D steps ahead, and the next k block's
    // weights are widened between the steps.
    constexpr int STEPS = 4 * MB, D = STEPS < 4 ? STEPS : 4, WPS = (NCB + MB - 1) / MB;
    f16x8 wv[2][NCB], av[D];
    auto widen = [&](int u, int c) __attribute__((always_inline)) {
      const f16x2 z1 = NG < 4 ? zero[NG < 4 ? u / GB : 0][c] : zero_of(u / GB, c);
      const f16x2 r1 = NG < 4 ? r[NG < 4 ? u / GB : 0][c] : scale_of(u / GB, c);
      wv[u & 1][c] = w4_widen_f16(t.w[c][u], bits, z1, z1 - f16x2{960, 960}, r1);
    };
    auto read = [&](int s) __attribute__((always_inline)) {
      av[s % D] = *reinterpret_cast<const f16x8*>(stage + s % MB * 4096 + (((4 * (s / MB) + lch) ^ lrow) * 16));
    };
#pragma unroll
    for (int s = 0; s < D; ++s) read(s);
#pragma unroll
    for (int c = 0; c < NCB; ++c) widen(0, c);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int u = s / MB, m = s % MB;
#pragma unroll
      for (int c = 0; c < NCB; ++c)
        acc[m][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(av[s % D], wv[u & 1][c], acc[m][c], 0, 0, 0);
      if (s + D < STEPS) read(s + D);
      if (u < 3) {
#pragma unroll
        for (int c = 0; c < NCB; ++c)
          if (MB < NCB ? c / WPS == m : c * MB / NCB == m) widen(u + 1, c);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // Set s: its codes were issued during set s - 1 and its activations during set s - NST + 1; each wave waits
  // for its own before the barrier that opens the set, which also ends all reads of the stage written next.
  // One body, and the codes handed on by register moves: a body for each half of an unrolled pair with an exit
  // between them spilled the accumulators.
  Weights w0, w1;
  load_w(kb_begin, w0);
#pragma unroll
  for (int i = 0; i < NST - 1; ++i) load_act(kb_begin + i * KS, i);
  int st = 0;
  for (int kb0 = kb_begin; kb0 < kb_end; kb0 += KS) {
    wait_vmcnt<(NST - 2) * ND>();
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    load_w(kb0 + KS, w1);
    __builtin_amdgcn_sched_barrier(0);
    load_act(kb0 + (NST - 1) * KS, st == 0 ? NST - 1 : st - 1);
    __builtin_amdgcn_sched_barrier(0);
    compute(st, w0);
    __builtin_amdgcn_sched_barrier(0);
    st = st + 1 == NST ? 0 : st + 1;
    w0 = w1;
  }
  wait_vmcnt<0>();
  __syncthreads();

  // Partial products of the k groups: row block t is finished by group t % KS.
  if constexpr (KS > 1) {
    f32x4* red = reinterpret_cast<f32x4*>(smem);
    auto red_at = [&](int g, int t, int c) {
      const int gi = g < t % KS ? g : g - 1;
      return ((((gi * WM + wm) * MB + t) * WN + wn) * NCB + c) * 64 + lane;
    };
#pragma unroll
    for (int t = 0; t < MB; ++t)
      if (t % KS != kg) {
#pragma unroll
        for (int c = 0; c < NCB; ++c) red[red_at(kg, t, c)] = acc[t][c];
      }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < MB; ++t)
      if (t % KS == kg) {
#pragma unroll
        for (int c = 0; c < NCB; ++c) {
          f32x4 v = t % KS == 0 ? acc[t][c] : red[red_at(0, t, c)];
#pragma unroll
          for (int g = 1; g < KS; ++g) v += g == t % KS ? acc[t][c] : red[red_at(g, t, c)];
          acc[t][c] = v;
        }
      }
    __syncthreads();
  }
  if (p.splits > 1) {
#pragma unroll
    for (int t = 0; t < MB; ++t) {
      if (t % KS != kg) continue;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = (wm * MB + t) * 16 + lch * 4 + r;
        if (row >= rows) continue;
        float* dst = p.partial + ((int64_t)split * p.M + m0 + row) * p.NP;
#pragma unroll
        for (int c = 0; c < NCB; ++c)
          if (cb0 + c < npb) dst[(cb0 + c) * 16 + lrow] = acc[t][c][r];
      }
    }
    return;
  }
  // Outputs through LDS, so that whole 16-byte pieces of rows are stored.
  __bf16* out = reinterpret_cast<__bf16*>(smem);
  const int n_tile = tile * OUTC;
#pragma unroll
  for (int t = 0; t < MB; ++t) {
    if (t % KS != kg) continue;
    const int row = (wm * MB + t) * 16 + lch * 4;
    float s[4], given[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[r] = row + r < rows ? p.factor[m0 + row + r] : 0.0f;
      given[r] = row + r < rows ? w4_given_scale<EPI>(p, m0 + row + r) : 0.0f;
    }
#pragma unroll
    for (int c = 0; c < NCB; c += STEP) {
      const int col = (wn * NCB + c) / STEP * 16 + lrow;
      const float bias = EPI == EPI_RMS && p.bias && n_tile + col < p.ncols ? p.bias[n_tile + col] : 0.0f;
      const float f0 = 1.0f / norm[c], f1 = 1.0f / norm[c + STEP - 1];
#pragma unroll
      for (int r = 0; r < 4; ++r)
        out[(row + r) * PITCH + col] =
            (__bf16)w4_many_value<EPI>(acc[t][c][r], acc[t][c + STEP - 1][r], f0, f1, s[r], given[r], bias);
    }
  }
  __syncthreads();
  for (int q = threadIdx.x; q < rows * (OUTC / 8); q += 64 * NW) {
    const int r = q / (OUTC / 8), n = n_tile + q % (OUTC / 8) * 8;
    const __bf16* src = out + r * PITCH + q % (OUTC / 8) * 8;
    __bf16* dst = p.y + (int64_t)(m0 + r) * p.ldy + n;
    if (n + 8 <= p.ncols) {
      store_out16(dst, *reinterpret_cast<const u32x4*>(src));
    } else {
      for (int e = 0; n + e < p.ncols; ++e) dst[e] = src[e];
    }
  }
}

// Joins the splits of K in order and applies the epilogue: one thread per four packed columns of a row (GLU:
// four gate columns and their up columns).  Bound by memory: two splits of 333 x 12288 9.3 us for 41 MB (12.0 with
// the outputs stored one by one).
template <int EPI>
__global__ __launch_bounds__(256) void w4_join_kernel(W4Gemm p) {
  constexpr int STEP = epi_is_glu(EPI) ? 2 : 1;
  const int quads = p.NP / (4 * STEP);
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t m = i / quads;
  const int n = (int)(i % quads) * 4;  // output column
  if (m >= p.M || n >= p.ncols) return;
  const int c = STEP == 2 ? n / 16 * 32 + n % 16 : n;
  f32x4 v = {0.f, 0.f, 0.f, 0.f}, u = v;
  for (int s0 = 0; s0 < p.splits; s0 += 8) {  // eight loads in flight
    f32x4 a[8], b[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      a[s] = b[s] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (s0 + s < p.splits) {
        const float* src = p.partial + ((int64_t)(s0 + s) * p.M + m) * p.NP + c;
        a[s] = *reinterpret_cast<const f32x4*>(src);
        if constexpr (STEP == 2) b[s] = *reinterpret_cast<const f32x4*>(src + 16);
      }
    }
#pragma unroll
    for (int s = 0; s < 8; ++s) v += a[s], u += b[s];
  }
  const float f = p.factor[m], given = w4_given_scale<EPI>(p, m);
  const f32x4 n0 = *reinterpret_cast<const f32x4*>(p.col_norm + c);
  f32x4 n1 = n0;
  if constexpr (STEP == 2) n1 = *reinterpret_cast<const f32x4*>(p.col_norm + c + 16);
  float o[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float bias = EPI == EPI_RMS && p.bias && n + e < p.ncols ? p.bias[n + e] : 0.0f;
    o[e] = w4_many_value<EPI>(v[e], u[e], 1.0f / n0[e], 1.0f / n1[e], f, given, bias);
  }
  __bf16* dst = p.y + m * p.ldy + n;
  if (n + 4 <= p.ncols) {
    *reinterpret_cast<u32x2*>(dst) = pack4_bf16(o);
  } else {
    for (int e = 0; n + e < p.ncols; ++e) dst[e] = (__bf16)o[e];
  }
}

// Rows from which the activations are staged: at 5 x 11008 -> 4096 the two are within 4% of each other.
constexpr int kW4StagedM = 6;

template <int NCB, int KS, int RG, int GB, int EPI, bool GS>
static hipError_t launch_w4_few_cfg(const W4Args& p) {
  const int tiles = (p.NP / 16 + NCB - 1) / NCB, groups = (p.M + 16 * RG - 1) / (16 * RG);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)tiles * groups), dim3(64 * KS), 0, p.stream, p.a, p.M, p.K, p.lda, p.codes,
                       p.scales, p.NP, p.KB, p.ncols, p.y, p.ldy, p.ep, groups);
    return hipGetLastError();
  };
  if constexpr (!GS && RG == 1)
    if (p.M < kW4StagedM) return go(w4_few_kernel<NCB, KS, RG, GB, EPI, GS, false>);
  return go(w4_few_kernel<NCB, KS, RG, GB, EPI, GS, true>);
}

// The shapes of w4_linear.hip's kW4Few, in its order.
template <int GB, int EPI, bool GS>
static hipError_t launch_w4_few_g(const W4Args& p, int shape) {
  switch (shape) {
    case 0: return launch_w4_few_cfg<2, 8, 1, GB, EPI, GS>(p);
    case 1: return launch_w4_few_cfg<4, 8, 1, GB, EPI, GS>(p);
    case 2: return launch_w4_few_cfg<6, 8, 1, GB, EPI, GS>(p);
    case 3: return launch_w4_few_cfg<4, 4, 1, GB, EPI, GS>(p);
    case 4: return launch_w4_few_cfg<2, 4, 1, GB, EPI, GS>(p);
  }
  if constexpr (!GS) {
    if (shape == 5) return launch_w4_few_cfg<4, 8, 2, GB, EPI, GS>(p);
    if constexpr (GB == 4)
      if (shape == 6) return launch_w4_few_cfg<6, 8, 2, GB, EPI, GS>(p);
  }
  if constexpr (!epi_is_glu(EPI)) {
    if (shape == 7) return launch_w4_few_cfg<1, 8, 1, GB, EPI, GS>(p);
    if constexpr (!GS)
      if (shape == 8) return launch_w4_few_cfg<1, 16, 1, GB, EPI, GS>(p);
    if (shape == 9) return launch_w4_few_cfg<3, 8, 1, GB, EPI, GS>(p);
  }
  return hipErrorInvalidValue;
}

template <int EPI>
hipError_t launch_w4_few(const W4Args& p, int shape) {
  auto go = [&](auto gb) {
    constexpr int GB = decltype(gb)::value;
    if constexpr (EPI != EPI_ROWSCALE)
      if (p.ep.g_rt) return launch_w4_few_g<GB, EPI, true>(p, shape);
    return launch_w4_few_g<GB, EPI, false>(p, shape);
  };
  if (p.group == 32) return go(std::integral_constant<int, 1>{});
  if (p.group == 64) return go(std::integral_constant<int, 2>{});
  return go(std::integral_constant<int, 4>{});
}

template <int MB, int NCB, int WN, int KS, int GB, int EPI>
static hipError_t launch_w4_many_cfg(const W4Gemm& q, hipStream_t stream) {
  const int tiles = (q.NP / 16 + NCB * WN - 1) / (NCB * WN);
  hipLaunchKernelGGL((w4_gemm_kernel<MB, NCB, 1, WN, KS, 2, GB, EPI>), dim3((unsigned)tiles * q.groups * q.splits),
                     dim3(64 * WN * KS), 0, stream, q);
  return hipGetLastError();
}

// The shapes of w4_linear.hip's kW4Many, in its order.
template <int GB, int EPI>
static hipError_t launch_w4_many_g(const W4Gemm& q, int shape, hipStream_t stream) {
  switch (shape) {
    case 0: return launch_w4_many_cfg<8, 4, 4, 1, GB, EPI>(q, stream);
    case 1: return launch_w4_many_cfg<8, 2, 4, 1, GB, EPI>(q, stream);
    case 2: return launch_w4_many_cfg<6, 4, 4, 1, GB, EPI>(q, stream);
    case 3: return launch_w4_many_cfg<6, 2, 4, 1, GB, EPI>(q, stream);
    case 4: return launch_w4_many_cfg<4, 2, 4, 2, GB, EPI>(q, stream);
    case 5: return launch_w4_many_cfg<4, 2, 4, 1, GB, EPI>(q, stream);
    case 6: return launch_w4_many_cfg<2, 2, 4, 2, GB, EPI>(q, stream);
    case 7: return launch_w4_many_cfg<2, 2, 2, 4, GB, EPI>(q, stream);
    case 8: return launch_w4_many_cfg<6, 2, 4, 2, GB, EPI>(q, stream);
    case 9: return launch_w4_many_cfg<8, 2, 4, 2, GB, EPI>(q, stream);
    case 10: return launch_w4_many_cfg<2, 2, 1, 8, GB, EPI>(q, stream);
  }
  return hipErrorInvalidValue;
}

template <int EPI>
hipError_t launch_w4_many(const W4Gemm& q, int group, int shape, hipStream_t stream) {
  const hipError_t e = group == 32   ? launch_w4_many_g<1, EPI>(q, shape, stream)
                       : group == 64 ? launch_w4_many_g<2, EPI>(q, shape, stream)
                                     : launch_w4_many_g<4, EPI>(q, shape, stream);
  if (e != hipSuccess || q.splits == 1) return e;
  const int64_t threads = (int64_t)q.M * (q.NP / (epi_is_glu(EPI) ? 8 : 4));
  hipLaunchKernelGGL(w4_join_kernel<EPI>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, q);
  return hipGetLastError();
}

}  // namespace fn
