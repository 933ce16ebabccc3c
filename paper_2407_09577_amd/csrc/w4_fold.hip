// 4-bit weights: quantising a weight with g folded in, packing codes that a checkpoint brings, and
// reading the weight back.  Off the hot path, once per weight.
#include "fn_fold.h"
#include "fn_launch.h"
#include "fn_w4.h"

namespace fn {

// s rounded to 12 significant bits, ties to even.
__device__ __forceinline__ double twelve_bits(double s) {
  unsigned long long u = (unsigned long long)__double_as_longlong(s);
  u += 0xffffffffffull + ((u >> 41) & 1ull);
  return __longlong_as_double((long long)(u & ~((1ull << 41) - 1ull)));
}

// One wave quantises a code fragment: lane 16 c + p holds 32 k of column p, so a group's smallest and
// largest product meet across the four lanes of a column.  g w is exact in fp64, the scale is rounded
// once from it and the code is the nearest one to the fp64 quotient, so the result does not depend on
// the order of anything.
template <typename T, int GB>
__global__ __launch_bounds__(256) void w4_fold_kernel(const T* __restrict__ W, int64_t sk, int64_t sn, int64_t K,
                                                      int64_t N, const float* __restrict__ g, int glu, bool vec,
                                                      bool gvec, bool zero_points, int NPB, int KB, int kgroups,
                                                      u32x4* __restrict__ codes, unsigned* __restrict__ scales) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane >> 4;
  const int cq = blockIdx.x / kgroups, kq = blockIdx.x % kgroups;
  const int cb = sk == 1 ? cq : 4 * cq + wave, kb = sk == 1 ? 4 * kq + wave : kq;
  if (cb >= NPB || kb >= KB) return;
  const int64_t n = logical_col((int64_t)cb * 16 + (lane & 15), N, glu);
  float w[4][8], gv[4][8];
#pragma unroll
  for (int u = 0; u < 4; ++u) load_k8(W, sk, sn, (int64_t)kb * kW4KB + 32 * u + 8 * c, n, K, vec, w[u]);
#pragma unroll
  for (int u = 0; u < 4; ++u) load_v8(g, (int64_t)kb * kW4KB + 32 * u + 8 * c, K, gvec, 1.0f, gv[u]);
  u32x4 out;
#pragma unroll
  for (int u0 = 0; u0 < 4; u0 += GB) {
    double lo = 0.0, hi = 0.0;
    bool bad = false;
#pragma unroll
    for (int u = u0; u < u0 + GB; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double t = n >= 0 ? (double)gv[u][e] * (double)w[u][e] : 0.0;
        lo = fmin(lo, t);
        hi = fmax(hi, t);
        bad |= !(fabs(t) <= 0x1p300);
      }
#pragma unroll
    for (int o = 16; o <= 32; o <<= 1) {
      lo = fmin(lo, __shfl_xor(lo, o));
      hi = fmax(hi, __shfl_xor(hi, o));
      bad |= __shfl_xor((int)bad, o) != 0;
    }
    double s = twelve_bits(zero_points ? (hi - lo) / 15.0 : fmax(-lo, hi) / 7.0);
    if (s < 0x1p-126) s = 0.0;
    if (!(s <= 0x1.fffffep127) || bad) s = __builtin_nan("");
    double z = 8.0;
    if (zero_points && s > 0.0) z = fmin(fmax(rint(-lo / s), 0.0), 15.0);
#pragma unroll
    for (int u = u0; u < u0 + GB; ++u) {
      unsigned word = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double t = n >= 0 ? (double)gv[u][e] * (double)w[u][e] : 0.0;
        const double q = s > 0.0 ? fmin(fmax(rint(t / s) + z, 0.0), 15.0) : z;
        word |= (unsigned)(int)q << w4_bit(e);
      }
      out[u] = word;
    }
    if (lane < 16)
      scales[((int64_t)kb * (4 / GB) + u0 / GB) * NPB * 16 + cb * 16 + lane] =
          (__float_as_uint((float)s) & kW4ScaleMask) | (unsigned)(int)z;
  }
  codes[((int64_t)kb * NPB + cb) * 64 + lane] = out;
}

__global__ __launch_bounds__(256) void w4_pack_kernel(const uint8_t* __restrict__ q, int64_t ldq,
                                                      const float* __restrict__ s, int64_t lds,
                                                      const uint8_t* __restrict__ z, int64_t ldz, int64_t K, int64_t N,
                                                      int glu, int gb, int NPB, int KB, u32x4* __restrict__ codes,
                                                      unsigned* __restrict__ scales) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane >> 4;
  const int kb = blockIdx.x % KB, cb = 4 * (blockIdx.x / KB) + wave;
  if (cb >= NPB) return;
  const int64_t n = logical_col((int64_t)cb * 16 + (lane & 15), N, glu);
  u32x4 out;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    unsigned word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int64_t k = (int64_t)kb * kW4KB + 32 * u + 8 * c + e;
      const unsigned v = n >= 0 && k < K ? q[k * ldq + n] & 15u : 0u;
      word |= v << w4_bit(e);
    }
    out[u] = word;
  }
  codes[((int64_t)kb * NPB + cb) * 64 + lane] = out;
  const int64_t groups = (K + 32 * gb - 1) / (32 * gb);
  if (c >= 4 / gb) return;  // lane 16 c + p writes group c of the fragment
  const int64_t grp = (int64_t)kb * (4 / gb) + c;
  unsigned word = 8u;
  if (n >= 0 && grp < groups) {
    unsigned b = __float_as_uint(s[grp * lds + n]);
    const bool nan = (b & 0x7fffffffu) > 0x7f800000u;
    b = nan ? 0x7fc00000u : (b + 0x7ffu + ((b >> 12) & 1u)) & kW4ScaleMask;
    word = b | (z ? z[grp * ldz + n] & 63u : 8u);
  }
  scales[grp * NPB * 16 + cb * 16 + (lane & 15)] = word;
}

// The power of two that brings a packed column's largest |s| into [2^9, 2^10): sixteen threads per column.
__global__ __launch_bounds__(256) void w4_norms_kernel(const unsigned* __restrict__ scales, int64_t groups, int64_t NP,
                                                       float* __restrict__ norms) {
  __shared__ unsigned red[16][16];
  const int c = threadIdx.x & 15, w = threadIdx.x >> 4;
  const int64_t col = (int64_t)blockIdx.x * 16 + c;
  unsigned top = 0;
#pragma unroll 4
  for (int64_t g = w; g < groups; g += 16) top = max(top, scales[g * NP + col] & 0x7ffff000u);
  red[w][c] = top;
  __syncthreads();
  if (w) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) top = max(top, red[i][c]);
  const unsigned ex = top >> 23;  // 255: a column that holds no finite scale stays as it is
  norms[col] = ex == 255u || top == 0u ? 1.0f : __uint_as_float(min(263u - ex, 254u) << 23);
}

static hipError_t launch_w4_norms(void* w4, int64_t K, int64_t N, int glu, int group, hipStream_t stream) {
  const int64_t NP = packed_cols(N, glu);
  hipLaunchKernelGGL(w4_norms_kernel, dim3((unsigned)(NP / 16)), dim3(256), 0, stream, w4_scales(w4, K, N, glu),
                     w4_blocks(K) * (128 / group), NP, w4_norms(w4, K, N, glu, group));
  return hipGetLastError();
}

// The weight that the codes stand for, in fp32 (exact: (q - z) has 9 bits, s 12).
__global__ __launch_bounds__(256) void w4_unpack_kernel(const u32x4* __restrict__ codes,
                                                        const unsigned* __restrict__ scales, int64_t K, int64_t N,
                                                        int glu, int gb, int NPB, int KB, float* __restrict__ out,
                                                        int64_t ldo) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane >> 4;
  const int kb = blockIdx.x % KB, cb = 4 * (blockIdx.x / KB) + wave;
  if (cb >= NPB) return;
  const int64_t n = logical_col((int64_t)cb * 16 + (lane & 15), N, glu);
  if (n < 0) return;
  const u32x4 words = codes[((int64_t)kb * NPB + cb) * 64 + lane];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const unsigned sw = scales[((int64_t)kb * (4 / gb) + u / gb) * NPB * 16 + cb * 16 + (lane & 15)];
    const float s = w4_scale(sw), z = w4_zero(sw);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int64_t k = (int64_t)kb * kW4KB + 32 * u + 8 * c + e;
      if (k < K) out[k * ldo + n] = ((float)((words[u] >> w4_bit(e)) & 15u) - z) * s;
    }
  }
}

template <typename T>
static hipError_t launch_w4_fold_t(const W4FoldArgs& p) {
  const T* W = reinterpret_cast<const T*>(p.W);
  auto aligned = [](const void* q) { return (reinterpret_cast<uintptr_t>(q) & 15) == 0; };
  const bool vec = p.sk == 1 && p.K % 8 == 0 && aligned(W) && p.sn * (int64_t)sizeof(T) % 16 == 0;
  const int NPB = (int)(packed_cols(p.N, p.glu) / 16), KB = (int)w4_blocks(p.K);
  const int kstep = p.sk == 1 ? 4 : 1, cstep = p.sk == 1 ? 1 : 4, kgroups = (KB + kstep - 1) / kstep;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)kgroups * ((NPB + cstep - 1) / cstep)), dim3(256), 0, p.stream, W, p.sk,
                       p.sn, p.K, p.N, p.g, p.glu, vec, aligned(p.g), p.zero_points, NPB, KB, kgroups,
                       reinterpret_cast<u32x4*>(p.w4), w4_scales(p.w4, p.K, p.N, p.glu));
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? launch_w4_norms(p.w4, p.K, p.N, p.glu, p.group, p.stream) : e;
  };
  return p.group == 32 ? go(w4_fold_kernel<T, 1>) : p.group == 64 ? go(w4_fold_kernel<T, 2>) : go(w4_fold_kernel<T, 4>);
}

hipError_t launch_w4_fold(const W4FoldArgs& p) {
  return p.w_dtype == kDtypeBf16 ? launch_w4_fold_t<unsigned short>(p) : launch_w4_fold_t<float>(p);
}

hipError_t launch_w4_pack(const uint8_t* codes, int64_t ldc, const float* scales, int64_t lds, const uint8_t* zeros,
                          int64_t ldz, int64_t K, int64_t N, int glu, int group, void* w4, hipStream_t stream) {
  const int NPB = (int)(packed_cols(N, glu) / 16), KB = (int)w4_blocks(K);
  hipLaunchKernelGGL(w4_pack_kernel, dim3((unsigned)KB * ((NPB + 3) / 4)), dim3(256), 0, stream, codes, ldc, scales, lds,
                     zeros, ldz, K, N, glu, group / 32, NPB, KB, reinterpret_cast<u32x4*>(w4), w4_scales(w4, K, N, glu));
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? launch_w4_norms(w4, K, N, glu, group, stream) : e;
}

hipError_t launch_w4_unpack(const void* w4, int64_t K, int64_t N, int glu, int group, float* out, int64_t ldo,
                            hipStream_t stream) {
  const int NPB = (int)(packed_cols(N, glu) / 16), KB = (int)w4_blocks(K);
  hipLaunchKernelGGL(w4_unpack_kernel, dim3((unsigned)KB * ((NPB + 3) / 4)), dim3(256), 0, stream,
                     reinterpret_cast<const u32x4*>(w4), w4_scales(const_cast<void*>(w4), K, N, glu), K, N, glu,
                     group / 32, NPB, KB, out, ldo);
  return hipGetLastError();
}

}  // namespace fn
