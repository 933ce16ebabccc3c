// 4-bit weights: quantising a weight with g folded in, packing codes that a checkpoint brings, and
// reading the weight back.  Off the hot path, once per weight.
#include <type_traits>

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

// A group's scale and zero point from its extremes, and the quotient -lo / s that z is rounded from (0 where there is
// none).  R(span) below 2^-126 is 0, beyond fp32 NaN; then z = 8.
__device__ __forceinline__ double w4_span(double lo, double hi, bool zero_points) {
  return zero_points ? (hi - lo) / 15.0 : fmax(-lo, hi) / 7.0;
}
__device__ __forceinline__ double w4_scale_of(double span, double lo, bool bad, bool zero_points, float& s, float& z) {
  const double d = twelve_bits(span);
  s = bad || !(d <= 0x1.fffffep127) ? __builtin_nanf("") : d < 0x1p-126 ? 0.0f : (float)d;
  const double at = zero_points && s > 0.0f ? -lo / d : 0.0;
  z = zero_points && s > 0.0f ? (float)fmin(fmax(rint(at), 0.0), 15.0) : 8.0f;
  return at;
}

// A weight view and the position of a lane's 32 values in it: k0 + 32 u + e.
template <typename T>
struct W4Source {
  const T* W;
  int64_t sk, sn, K, n, k0;
  const float* g;
  bool vec, gvec;
  // Eight products g w, rounded to fp32; zeros past K.
  __device__ __forceinline__ void products(int u, float (&p)[8]) const {
    float gv[8];
    load_k8(W, sk, sn, k0 + 32 * u, n, K, vec, p);
    load_v8(g, k0 + 32 * u, K, gvec, 1.0f, gv);
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] *= gv[e];
  }
  // The same from a fragment that lies in LDS, [128][16].
  __device__ __forceinline__ void products(const T* own, int u, float (&p)[8]) const {
    float gv[8];
    load_v8(g, k0 + 32 * u, K, gvec, 1.0f, gv);
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = widen(own[(32 * u + e) * 16]) * gv[e];
  }
  // One product, exactly.
  __device__ __forceinline__ double exact(int u, int e) const {
    const int64_t k = k0 + 32 * u + e;
    if (n < 0 || k >= K) return 0.0;
    return (double)widen(W[k * sk + n * sn]) * (g ? (double)g[k] : 1.0);
  }
};

__device__ __forceinline__ void w4_put(u32x4& out, int u, int e, unsigned q) {
  const unsigned shift = w4_bit(e);
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = i == u ? (out[i] & ~(15u << shift)) | q << shift : out[i];
}

// The power of two that brings a largest |s| with these bits into [2^9, 2^10).
__device__ __forceinline__ float w4_norm_of(unsigned top) {
  const unsigned ex = top >> 23;  // 255: a column that holds no finite scale stays as it is
  return ex == 255u || top == 0u ? 1.0f : __uint_as_float(min(263u - ex, 254u) << 23);
}

// One wave quantises a code fragment: lane 16 c + p holds 32 k of column p, so a group's smallest and largest
// product meet across the four lanes of a column.  By definition g w is exact, the scale is rounded once from
// the extremes and the code is the nearest one to the fp64 quotient, so the result does not depend on the order
// of anything.  fp32 decides the same nearly always:
//   the extremes and the span are off by at most 2^-24 of themselves, so the scale is the exact one's unless a
//   border between twelve-bit values lies that near (one group in 1000: the products that round to the extremes
//   are taken again in fp64);
//   the zero point's quotient -lo / s (at most 15 and a bit), by that scale, is off by 2^-24 of itself, less than
//   2^-19, so it rounds to the right one unless it is that near to a half (then again in fp64);
//   a quotient (at most 16) is off by 3 * 2^-24 of itself, less than 2^-18, so its nearest whole number is the
//   right one unless it is that near to a half (one weight in 130000: decided again in fp64).
// Groups whose largest product is not between 2^-100 and 2^100 are taken in fp64 throughout, but for zeros.
// A wave loads its fragment, waits and computes, 22 vector operations a weight, so neither memory nor the vector units
// are busy for more than six tenths of the time.  4096 x 22016 bf16 from [N, K]: 114 us with fp64 quotients throughout,
// 65 to 90 us so (on different cards), for 228 MB.
// A workgroup takes cw column and kw k blocks.  Of the four lanes of a column each makes the scale of one group, if
// there are as many: made by each lane in turn, four groups' fp64 took 3 us of a small fold and a fifth of a large
// one (4096 x 22016, groups of 32: 91 us a call, 71 so).  WHOLE: kw is all of K, so the workgroup sees whole columns
// and writes their norms too, and no second launch reads the scales (576 x 1536: 12.2 us a call in all, 8.1 so).
template <typename T, int GB, bool WHOLE, bool ROWS>
__global__ __launch_bounds__(WHOLE ? 1024 : 256) void w4_fold_kernel(
    const T* __restrict__ W, int64_t sk, int64_t sn, int64_t K, int64_t N, const float* __restrict__ g, int glu, bool vec,
    bool gvec, bool zero_points, int NPB, int KB, int cw, int kw, int kgroups, u32x4* __restrict__ codes,
    unsigned* __restrict__ scales, float* __restrict__ norms) {
  constexpr int NG = 4 / GB;
  __shared__ unsigned tops[WHOLE ? 16 : 1][16];
  const int lane = threadIdx.x & 63, c = lane >> 4, p16 = lane & 15;
  const int wave = WHOLE ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : threadIdx.x >> 6;
  const int cq = blockIdx.x / kgroups, kq = blockIdx.x % kgroups;
  const int cb = WHOLE ? cq * cw + wave % cw : cw == 1 ? cq : 4 * cq + wave;
  const int kb = WHOLE ? wave / cw : cw == 1 ? 4 * kq + wave : kq;
  const bool live = cb < NPB && kb < KB;  // else zeros, which only the barrier needs
  if (!WHOLE && !live) return;
  const W4Source<T> src{W, sk, sn, K, logical_col((int64_t)cb * 16 + p16, N, glu), (int64_t)kb * kW4KB + 8 * c, g, vec,
                        gvec};
  // ROWS, bf16 with unit column stride: runs of 16 bytes of a row through LDS, each wave its own fragment (zeros past K
  // and the columns).  4096 x 11008 in rows 40.7 us with a load for each value, 34.3 so; in fp32, where such loads
  // bring twice the bytes, the two are within 5% of each other either way.
  constexpr int EL = 16 / sizeof(T), RUNS = 16 / EL;
  __shared__ __align__(16) T stage[ROWS ? (WHOLE ? 16 : 4) : 1][ROWS ? kW4KB * 16 : 1];
  if constexpr (ROWS) {
    const int64_t n = logical_col((int64_t)cb * 16, N, glu);
    const int64_t left = n < 0 ? 0 : (glu && n < N / 2 ? N / 2 : N) - n;
    const int run = lane % RUNS;
    u32x4 v[2 * RUNS];
#pragma unroll
    for (int i = 0; i < 2 * RUNS; ++i) {
      const int row = i * (64 / RUNS) + lane / RUNS;
      const int64_t k = (int64_t)kb * kW4KB + row;
      const T* from = W + k * sk + n + run * EL;
      v[i] = u32x4{0, 0, 0, 0};
      if (k < K && left >= (run + 1) * EL) {
        __builtin_memcpy(&v[i], from, 16);
      } else if (k < K) {
        T t[EL];
#pragma unroll
        for (int e = 0; e < EL; ++e) t[e] = run * EL + e < left ? from[e] : T(0);
        __builtin_memcpy(&v[i], t, 16);
      }
    }
#pragma unroll
    for (int i = 0; i < 2 * RUNS; ++i)
      *reinterpret_cast<u32x4*>(&stage[wave][(i * (64 / RUNS) + lane / RUNS) * 16 + run * EL]) = v[i];
    wave_lds_order();
  }
  const int mine = c & (NG - 1);
  float p[4][8], low[NG], high[NG], lo_m = 0.0f, hi_m = 0.0f, any_m = 0.0f;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if constexpr (ROWS) src.products(stage[wave] + 8 * c * 16 + p16, u, p[u]);
    else src.products(u, p[u]);
  }
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    float lo = 0.0f, hi = 0.0f, any = 0.0f;
#pragma unroll
    for (int u = j * GB; u < (j + 1) * GB; ++u)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        lo = fminf(fminf(lo, p[u][e]), p[u][e + 1]);
        hi = fmaxf(fmaxf(hi, p[u][e]), p[u][e + 1]);
        any += p[u][e] + p[u][e + 1];  // NaN where a product is: the extremes skip it
      }
#pragma unroll
    for (int o = 16; o <= 32; o <<= 1) {
      lo = fminf(lo, __shfl_xor(lo, o));
      hi = fmaxf(hi, __shfl_xor(hi, o));
      any += __shfl_xor(any, o);
    }
    low[j] = lo, high[j] = hi;
    if (j == mine) lo_m = lo, hi_m = hi, any_m = any;
  }
  const double span = w4_span(lo_m, hi_m, zero_points);
  const float top = fmaxf(-lo_m, hi_m);
  float s_m, z_m;
  const double at_m = w4_scale_of(span, lo_m, false, zero_points, s_m, z_m);
  const bool far_m = any_m != any_m || !(top == 0.0f || (top >= 0x1p-100f && top <= 0x1p100f));
  const bool near_m =
      top > 0.0f && (twelve_bits(span * (1.0 - 0x1p-23)) != twelve_bits(span * (1.0 + 0x1p-23)) ||
                     fabs(at_m - rint(at_m)) > 0.5 - 0x1p-19);
  if (__any(near_m | far_m)) {
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      if (!__any(mine == j && (near_m | far_m))) continue;
      // Rounding keeps the order: the exact extremes are among the products that round to the extremes.
      unsigned at = (NG == 1 ? (int)far_m : __shfl((int)far_m, p16 + 16 * j)) ? 0xffffffffu : 0;
#pragma unroll
      for (int u = j * GB; u < (j + 1) * GB; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (p[u][e] == low[j] || p[u][e] == high[j]) at |= 1u << (8 * u + e);
      if constexpr (GB < 4) at &= ((1u << (8 * (GB & 3))) - 1u) << (8 * GB * j);
      double lo = 0.0, hi = 0.0;
      bool bad = false;
      while (at) {
        const int i = __builtin_ctz(at);
        at &= at - 1;
        const double t = src.exact(i >> 3, i & 7);
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
      float sj, zj;
      w4_scale_of(w4_span(lo, hi, zero_points), lo, bad, zero_points, sj, zj);
      if (j == mine) s_m = sj, z_m = zj;
    }
  }
  float s[NG], z[NG];
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    s[j] = NG == 1 ? s_m : __shfl(s_m, p16 + 16 * j);
    z[j] = NG == 1 ? z_m : __shfl(z_m, p16 + 16 * j);
  }
  int far = far_m;
  if constexpr (NG > 1) far |= __shfl_xor(far, 16);
  if constexpr (NG > 2) far |= __shfl_xor(far, 32);
  u32x4 out;
  unsigned again = 0;  // bit 8 u + e: the code is to be decided in fp64
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const float sj = s[u / GB], zj = z[u / GB], inv = sj > 0.0f ? 1.0f / sj : 0.0f;
    float q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float t = p[u][e] * inv, r = rintf(t);
      if (fabsf(t - r) > 0.5f - 0x1p-18f) again |= 1u << (8 * u + e);
      q[e] = r + zj;
      if (zero_points) q[e] = fminf(q[e], 15.0f);  // without them |r| is at most 7
    }
    // Codes to bytes (below zero: zero), even nibbles and odd ones.
    unsigned even = 0, odd = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = 4 * (i & 1) + (i >> 1);  // bytes 0..3: codes 0, 4, 1, 5; and 2, 6, 3, 7
      even = __builtin_amdgcn_cvt_pk_u8_f32(q[e], i, even);
      odd = __builtin_amdgcn_cvt_pk_u8_f32(q[e + 2], i, odd);
    }
    out[u] = even | odd << 4;
  }
  if (far) again = 0xffffffffu;
  while (again) {
    const int i = __builtin_ctz(again), u = i >> 3, e = i & 7;
    again &= again - 1;
    float sj = s[0], zj = z[0];
#pragma unroll
    for (int j = 1; j < NG; ++j)
      if (u / GB == j) sj = s[j], zj = z[j];
    const double q = sj > 0.0f ? fmin(fmax(rint(src.exact(u, e) / (double)sj) + (double)zj, 0.0), 15.0) : (double)zj;
    w4_put(out, u, e, (unsigned)(int)q);
  }
  const unsigned word = (__float_as_uint(s_m) & kW4ScaleMask) | (unsigned)z_m;
  if (live) {
    if (c < NG) scales[((int64_t)kb * NG + c) * NPB * 16 + cb * 16 + p16] = word;
    codes[((int64_t)kb * NPB + cb) * 64 + lane] = out;
  }
  if constexpr (WHOLE) {
    unsigned most = word & 0x7ffff000u;
    most = max(most, (unsigned)__shfl_xor((int)most, 16));
    most = max(most, (unsigned)__shfl_xor((int)most, 32));
    if (lane < 16) tops[wave][lane] = most;
    __syncthreads();
    if (wave >= cw || lane >= 16 || cb >= NPB) return;
    for (int k = 1; k < kw; ++k) most = max(most, tops[k * cw + wave][lane]);
    norms[cb * 16 + lane] = w4_norm_of(most);
  }
}

// One workgroup packs the fragments of one k block and eight column blocks: the codes come in runs of sixteen columns
// through LDS, where each wave picks its fragment's.  Bound by memory: 4096 x 22016 30 us with the
// norms, for 140 MB (77 us with every byte loaded where it is needed).
__global__ __launch_bounds__(512) void w4_pack_kernel(const uint8_t* __restrict__ q, int64_t ldq,
                                                      const float* __restrict__ s, int64_t lds,
                                                      const uint8_t* __restrict__ z, int64_t ldz, int64_t K, int64_t N,
                                                      int glu, int gb, int NPB, int KB, u32x4* __restrict__ codes,
                                                      unsigned* __restrict__ scales) {
  constexpr int PITCH = 128 + 16;
  __shared__ __align__(16) uint8_t tile[kW4KB * PITCH];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane >> 4;
  const int kb = blockIdx.x % KB, cb0 = 8 * (blockIdx.x / KB);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = i * 64 + threadIdx.x / 8, run = threadIdx.x % 8;
    const int64_t k = (int64_t)kb * kW4KB + row, n = logical_col((int64_t)(cb0 + run) * 16, N, glu);
    const int64_t left = n < 0 || k >= K ? 0 : (glu && n < N / 2 ? N / 2 : N) - n;  // columns of the run
    const uint8_t* src = q + k * ldq + n;
    u32x4 v = {0, 0, 0, 0};
    if (left >= 16) {
      __builtin_memcpy(&v, src, 16);  // rows start at any byte
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (e < left) v[e / 4] |= (unsigned)src[e] << (8 * (e % 4));
    }
    *reinterpret_cast<u32x4*>(tile + row * PITCH + 16 * run) = v;
  }
  __syncthreads();
  const int cb = cb0 + wave;
  if (cb >= NPB) return;
  const uint8_t* own = tile + 16 * wave + (lane & 15);
  u32x4 out;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    unsigned word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) word |= (unsigned)(own[(32 * u + 8 * c + e) * PITCH] & 15u) << w4_bit(e);
    out[u] = word;
  }
  codes[((int64_t)kb * NPB + cb) * 64 + lane] = out;
  const int64_t n = logical_col((int64_t)cb * 16 + (lane & 15), N, glu);
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

// The norms of columns whose scales other launches or workgroups wrote: sixteen threads per column, 1.6 to 4 us.
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
  norms[col] = w4_norm_of(top);
}

static hipError_t launch_w4_norms(void* w4, int64_t K, int64_t N, int glu, int group, hipStream_t stream) {
  const int64_t NP = packed_cols(N, glu);
  hipLaunchKernelGGL(w4_norms_kernel, dim3((unsigned)(NP / 16)), dim3(256), 0, stream, w4_scales(w4, K, N, glu),
                     w4_blocks(K) * (128 / group), NP, w4_norms(w4, K, N, glu, group));
  return hipGetLastError();
}

// The weight that the codes stand for, in fp32 (exact: (q - z) has 7 bits, s 12).  Bound by its stores: 4096 x 22016
// 77 us for 361 MB.
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
  // A workgroup takes all blocks of k where sixteen waves have room for them (beside two column blocks where the columns
  // lie together: with one, 2048 x 8192 in rows took 30.9 us, 18.9 in two launches).  Else four blocks along the
  // contiguous axis.
  const bool whole = KB <= (p.sk == 1 ? 16 : 8);
  const int cw = p.sk == 1 ? 1 : !whole || KB <= 4 ? 4 : 2, kw = whole ? KB : p.sk == 1 ? 4 : 1;
  const int kgroups = (KB + kw - 1) / kw;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)kgroups * ((NPB + cw - 1) / cw)), dim3(64 * cw * kw), 0, p.stream, W, p.sk,
                       p.sn, p.K, p.N, p.g, p.glu, vec, aligned(p.g), p.zero_points, NPB, KB, cw, kw, kgroups,
                       reinterpret_cast<u32x4*>(p.w4), w4_scales(p.w4, p.K, p.N, p.glu),
                       w4_norms(p.w4, p.K, p.N, p.glu, p.group));
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || whole ? e : launch_w4_norms(p.w4, p.K, p.N, p.glu, p.group, p.stream);
  };
  auto pick = [&](auto gb) {
    constexpr int GB = decltype(gb)::value;
    if constexpr (sizeof(T) == 2)
      if (p.sk != 1 && p.sn == 1)
        return whole ? go(w4_fold_kernel<T, GB, true, true>) : go(w4_fold_kernel<T, GB, false, true>);
    return whole ? go(w4_fold_kernel<T, GB, true, false>) : go(w4_fold_kernel<T, GB, false, false>);
  };
  if (p.group == 32) return pick(std::integral_constant<int, 1>{});
  return p.group == 64 ? pick(std::integral_constant<int, 2>{}) : pick(std::integral_constant<int, 4>{});
}

hipError_t launch_w4_fold(const W4FoldArgs& p) {
  return p.w_dtype == kDtypeBf16 ? launch_w4_fold_t<unsigned short>(p) : launch_w4_fold_t<float>(p);
}

hipError_t launch_w4_pack(const uint8_t* codes, int64_t ldc, const float* scales, int64_t lds, const uint8_t* zeros,
                          int64_t ldz, int64_t K, int64_t N, int glu, int group, void* w4, hipStream_t stream) {
  const int NPB = (int)(packed_cols(N, glu) / 16), KB = (int)w4_blocks(K);
  hipLaunchKernelGGL(w4_pack_kernel, dim3((unsigned)KB * ((NPB + 7) / 8)), dim3(512), 0, stream, codes, ldc, scales, lds,
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
