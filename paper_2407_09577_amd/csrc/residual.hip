// Block residual: what joins a block's output x to the residual stream h and leads into the next block,
//   z = x rsqrt(eps_post + mean x^2) g_post      (z = x without g_post)
//   H = res_scale h + branch_scale gate z
//   n = H rsqrt(eps_pre + mean H^2) g_pre
// and its gradients.  Memory-bound: each row is read once, held in registers between its sums, and
// written once.
#include "fn_device.h"
#include "fn_epilogue.h"
#include "fn_launch.h"

namespace fn {

namespace {

// 16 bytes of a row, widened to fp32.
template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
  u32x4 w;
  __device__ __forceinline__ float operator[](int i) const {
    if constexpr (sizeof(T) == 2) return (i & 1) ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]);
    else return __uint_as_float(w[i]);
  }
  __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const u32x4*>(p); }
};

template <typename T>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[16 / sizeof(T)]) {
  if constexpr (sizeof(T) == 2) {
    const u32x2 lo = pack4_bf16(*reinterpret_cast<const float(*)[4]>(v));
    const u32x2 hi = pack4_bf16(*reinterpret_cast<const float(*)[4]>(v + 4));
    *reinterpret_cast<u32x4*>(p) = u32x4{lo[0], lo[1], hi[0], hi[1]};
  } else {
    *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  }
}

template <int N>
__device__ __forceinline__ void load_f32(const float* p, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const f32x4 t = *reinterpret_cast<const f32x4*>(p + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[i + e] = t[e];
  }
}

// Sums of NV values over the TPR threads of a row, the same in all of them and in a fixed order.  One wave
// exchanges within itself; more meet in LDS, in the two halves of buf by turns, so one barrier a call
// is enough: a wave writes a half again only after the barrier of the call between.
template <int TPR, int NV>
__device__ __forceinline__ void row_sum(float (&v)[NV], float (*buf)[TPR / 64][NV], int& turn) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1)
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] += __shfl_xor(v[i], o);
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) buf[turn][threadIdx.x >> 6][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      v[i] = buf[turn][0][i];
#pragma unroll
      for (int w = 1; w < TPR / 64; ++w) v[i] += buf[turn][w][i];
    }
    turn ^= 1;
  }
}

// One workgroup of TPR threads per row, V vectors of 16 bytes per thread.
template <typename T, int TPR, int V>
__global__ __launch_bounds__(TPR) void residual_kernel(ResidualArgs p) {
  constexpr int VN = Vec<T>::N;
  __shared__ float buf[2][TPR / 64][1];
  int turn = 0;
  const int K = p.K;
  const float inv_k = 1.0f / (float)K;
  for (int64_t m = blockIdx.x; m < p.M; m += gridDim.x) {
    const T* xr = (const T*)p.x + m * p.ldx;
    const T* hr = (const T*)p.h + m * p.ldh;
    const T* gr = p.gate ? (const T*)p.gate + (int64_t)(m / p.gate_rows) * p.ldg : nullptr;
    float H[V][VN];
    Vec<T> x[V], h[V];
    float ss[1] = {0.f};
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int k = (j * TPR + threadIdx.x) * VN;
      x[j].w = h[j].w = u32x4{0, 0, 0, 0};
      if (k < K) {
        x[j].load(xr + k);
        h[j].load(hr + k);
      }
#pragma unroll
      for (int e = 0; e < VN; ++e) ss[0] = fmaf(x[j][e], x[j][e], ss[0]);
    }
    float sc = p.branch_scale;
    if (p.g_post) {
      row_sum<TPR, 1>(ss, buf, turn);
      sc *= rsqrtf(fmaf(ss[0], inv_k, p.eps_post));
    }
    float sh[1] = {0.f};
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int k = (j * TPR + threadIdx.x) * VN;
#pragma unroll
      for (int e = 0; e < VN; ++e) H[j][e] = 0.f;
      if (k >= K) continue;
      float w[VN];
#pragma unroll
      for (int e = 0; e < VN; ++e) w[e] = sc;
      if (p.g_post) {
        float g[VN];
        load_f32(p.g_post + k, g);
#pragma unroll
        for (int e = 0; e < VN; ++e) w[e] *= g[e];
      }
      if (gr) {
        Vec<T> g;
        g.load(gr + k);
#pragma unroll
        for (int e = 0; e < VN; ++e) w[e] *= g[e];
      }
#pragma unroll
      for (int e = 0; e < VN; ++e) {
        H[j][e] = fmaf(w[e], x[j][e], p.res_scale * h[j][e]);
        sh[0] = fmaf(H[j][e], H[j][e], sh[0]);
      }
      store_vec<T>((T*)p.out + m * p.ldo + k, H[j]);
    }
    if (!p.normed && !p.inv_rms) continue;
    row_sum<TPR, 1>(sh, buf, turn);
    const float r = rsqrtf(fmaf(sh[0], inv_k, p.eps_pre));
    if (p.inv_rms && threadIdx.x == 0) p.inv_rms[m] = r;
    if (!p.normed) continue;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int k = (j * TPR + threadIdx.x) * VN;
      if (k >= K) continue;
      float g[VN];
      load_f32(p.g_pre + k, g);
#pragma unroll
      for (int e = 0; e < VN; ++e) g[e] *= H[j][e] * r;
      store_vec<T>((T*)p.normed + m * p.ldn + k, g);
    }
  }
}

// How the backward pass cuts the rows into units, each one workgroup's: ranges of rows that hold whole
// gate segments (seg_per_unit > 0, dgate written by the unit) or lie in one (pieces per segment, dgate
// from partial sums).  Without a gate, or with one per row, the rows are cut evenly.
struct Units {
  int64_t count;
  int rows;          // rows of a unit
  int pieces;        // units per segment; 0: units hold whole segments or there is no sum over rows
};

Units units_of(int64_t M, int64_t gate_rows, bool gate) {
  const int64_t kUnits = 1024;
  if (M == 0) return Units{0, 0, 0};
  int64_t rows = (M + kUnits - 1) / kUnits;
  if (!gate || gate_rows == 1) return Units{(M + rows - 1) / rows, (int)rows, 0};
  const int64_t segs = (M + gate_rows - 1) / gate_rows, T = gate_rows < M ? gate_rows : M;
  if (T <= rows) {
    rows = rows / T * T;
    return Units{(M + rows - 1) / rows, (int)rows, 0};
  }
  const int64_t pieces = (T + rows - 1) / rows;
  rows = (T + pieces - 1) / pieces;
  return Units{segs * pieces, (int)rows, (int)pieces};
}

// Gradients of a unit's rows.  With p = rsqrt(eps_post + mean x^2), r = rsqrt(eps_pre + mean H^2),
// a = dn g_pre and v = branch_scale gate g_post x:
//   D  = dH + r (a - H r t),  t = r sum(a H) / K           the gradient at H
//   dh = res_scale D,  dx = p (branch_scale gate g_post D - x p q),  q = p sum(v D) / K
// and sum(v D) = sum(v dH) + r (sum(v a) - r t sum(v H)), so the five sums that D and dx need are taken
// in one pass over the row in registers, after the first one (p).
template <typename T, int TPR, int V>
__global__ __launch_bounds__(TPR) void residual_bwd_kernel(ResidualArgs p, Units un, float* part_post, float* part_pre,
                                                           float* part_gate) {
  constexpr int VN = Vec<T>::N;
  __shared__ float buf1[2][TPR / 64][1];
  __shared__ float buf5[2][TPR / 64][5];
  int turn1 = 0, turn5 = 0;
  const int K = p.K;
  const float inv_k = 1.0f / (float)K;
  const int64_t u = blockIdx.x;
  int64_t m0, m1;
  if (un.pieces) {
    const int64_t seg = u / un.pieces, s0 = seg * p.gate_rows;
    m0 = s0 + (u % un.pieces) * un.rows;
    m1 = min(min(m0 + un.rows, s0 + (int64_t)p.gate_rows), (int64_t)p.M);
  } else {
    m0 = u * un.rows;
    m1 = min(m0 + un.rows, (int64_t)p.M);
  }
  float gpost[V][VN], gpre[V][VN], apost[V][VN], apre[V][VN], agate[V][VN];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int k = (j * TPR + threadIdx.x) * VN;
#pragma unroll
    for (int e = 0; e < VN; ++e) gpost[j][e] = 1.0f, gpre[j][e] = apost[j][e] = apre[j][e] = agate[j][e] = 0.0f;
    if (k < K && p.g_post) load_f32(p.g_post + k, gpost[j]);
    if (k < K && p.g_pre) load_f32(p.g_pre + k, gpre[j]);
  }
  for (int64_t m = m0; m < m1; ++m) {
    Vec<T> x[V], h[V], gate[V], dho[V], dn[V];
    float ss[1] = {0.f};
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int k = (j * TPR + threadIdx.x) * VN;
      x[j].w = h[j].w = gate[j].w = dho[j].w = dn[j].w = u32x4{0, 0, 0, 0};
      if (k < K) {
        x[j].load((const T*)p.x + m * p.ldx + k);
        h[j].load((const T*)p.h + m * p.ldh + k);
        if (p.gate) gate[j].load((const T*)p.gate + m / p.gate_rows * p.ldg + k);
        if (p.dh_out) dho[j].load((const T*)p.dh_out + m * p.lddo + k);
        if (p.dn) dn[j].load((const T*)p.dn + m * p.lddn + k);
      }
#pragma unroll
      for (int e = 0; e < VN; ++e) ss[0] = fmaf(x[j][e], x[j][e], ss[0]);
    }
    float rp = 1.0f;
    if (p.g_post) {
      row_sum<TPR, 1>(ss, buf1, turn1);
      rp = rsqrtf(fmaf(ss[0], inv_k, p.eps_post));
    }
    float s5[5] = {0.f, 0.f, 0.f, 0.f, 0.f};  // H^2, a H, v dH, v a, v H
    auto scale_at = [&](int j, int e) { return p.gate ? p.branch_scale * gate[j][e] : p.branch_scale; };
    auto H_at = [&](int j, int e) {
      return fmaf(scale_at(j, e) * gpost[j][e] * rp, x[j][e], p.res_scale * h[j][e]);
    };
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int e = 0; e < VN; ++e) {
        const float H = H_at(j, e), a = dn[j][e] * gpre[j][e], v = scale_at(j, e) * gpost[j][e] * x[j][e];
        s5[0] = fmaf(H, H, s5[0]);
        s5[1] = fmaf(a, H, s5[1]);
        s5[2] = fmaf(v, dho[j][e], s5[2]);
        s5[3] = fmaf(v, a, s5[3]);
        s5[4] = fmaf(v, H, s5[4]);
      }
    row_sum<TPR, 5>(s5, buf5, turn5);
    const float r = p.g_pre ? rsqrtf(fmaf(s5[0], inv_k, p.eps_pre)) : 0.0f;
    const float t = r * s5[1] * inv_k;
    const float q = rp * (s5[2] + r * (s5[3] - r * t * s5[4])) * inv_k;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int k = (j * TPR + threadIdx.x) * VN;
      if (k >= K) continue;
      float odx[VN], odh[VN], og[VN];
#pragma unroll
      for (int e = 0; e < VN; ++e) {
        const float H = H_at(j, e), a = dn[j][e] * gpre[j][e], sc = scale_at(j, e);
        const float D = p.g_pre ? fmaf(r, fmaf(-(H * r), t, a), dho[j][e]) : dho[j][e];
        const float xp = x[j][e] * rp, dz = sc * D;
        odh[e] = p.res_scale * D;
        odx[e] = p.g_post ? rp * fmaf(-xp, q, dz * gpost[j][e]) : dz;
        og[e] = p.branch_scale * D * xp * gpost[j][e];
        apost[j][e] = fmaf(dz, xp, apost[j][e]);
        apre[j][e] = fmaf(dn[j][e], H * r, apre[j][e]);
        agate[j][e] += og[e];
      }
      store_vec<T>((T*)p.dx + m * p.lddx + k, odx);
      store_vec<T>((T*)p.dh + m * p.lddh + k, odh);
    }
    // The gate row's sum, where the unit holds all of its rows.
    if (p.dgate && !un.pieces && (m + 1 == m1 || (m + 1) % p.gate_rows == 0)) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int k = (j * TPR + threadIdx.x) * VN;
        if (k < K) store_vec<T>((T*)p.dgate + m / p.gate_rows * p.lddg + k, agate[j]);
#pragma unroll
        for (int e = 0; e < VN; ++e) agate[j][e] = 0.0f;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int k = (j * TPR + threadIdx.x) * VN;
    if (k >= K) continue;
#pragma unroll
    for (int i = 0; i < VN; i += 4) {
      const int64_t at = u * K + k + i;
      if (part_post)
        *reinterpret_cast<f32x4*>(part_post + at) = f32x4{apost[j][i], apost[j][i + 1], apost[j][i + 2], apost[j][i + 3]};
      if (part_pre)
        *reinterpret_cast<f32x4*>(part_pre + at) = f32x4{apre[j][i], apre[j][i + 1], apre[j][i + 2], apre[j][i + 3]};
      if (part_gate)
        *reinterpret_cast<f32x4*>(part_gate + at) = f32x4{agate[j][i], agate[j][i + 1], agate[j][i + 2], agate[j][i + 3]};
    }
  }
}

// Sums of the units' partials in a fixed order: out[s][k] = sum over the `count` units of segment s.
template <typename T>
__global__ __launch_bounds__(1024) void residual_reduce_kernel(const float* __restrict__ part, int K, int64_t count,
                                                               T* __restrict__ out, int64_t ldo) {
  __shared__ float red[16][64];
  const int k = blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
  const int64_t seg = blockIdx.y;
  float s = 0.f;
  if (k < K)
    for (int64_t u = w; u < count; u += 16) s += part[(seg * count + u) * K + k];
  red[w][threadIdx.x & 63] = s;
  __syncthreads();
  if (w == 0 && k < K) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += red[i][threadIdx.x];
    if constexpr (sizeof(T) == 2) out[seg * ldo + k] = (T)s;
    else out[seg * ldo + k] = s;
  }
}

// Threads per row and vectors per thread: K <= threads * vectors * (16 bytes).
template <typename T, typename F>
hipError_t with_shape(int K, F go) {
  const int n = (K + Vec<T>::N - 1) / Vec<T>::N;  // vectors of a row
  if (n <= 64) return go(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  if (n <= 128) return go(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{});
  if (n <= 256) return go(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
  if (n <= 512) return go(std::integral_constant<int, 512>{}, std::integral_constant<int, 1>{});
  if (n <= 1024) return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
  if (n <= 2048) return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
  return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 4>{});
}

template <typename T>
hipError_t launch_fwd_t(const ResidualArgs& p) {
  return with_shape<T>(p.K, [&](auto tpr, auto v) {
    constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value;
    if constexpr (sizeof(T) == 2 && V > 2) return hipErrorInvalidValue;
    else {
      hipLaunchKernelGGL((residual_kernel<T, TPR, V>), dim3(min(p.M, 1 << 20)), dim3(TPR), 0, p.stream, p);
      return hipGetLastError();
    }
  });
}

template <typename T>
hipError_t launch_bwd_t(const ResidualArgs& p) {
  const Units un = units_of(p.M, p.gate_rows, p.dgate != nullptr);
  float* next = p.ws;
  auto take = [&](bool wanted) {
    float* q = wanted ? next : nullptr;
    if (wanted) next += un.count * p.K;
    return q;
  };
  float* part_post = take(p.dg_post != nullptr);
  float* part_pre = take(p.dg_pre != nullptr);
  float* part_gate = take(p.dgate && un.pieces);
  const hipError_t e = with_shape<T>(p.K, [&](auto tpr, auto v) {
    constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value;
    if constexpr (sizeof(T) == 2 && V > 2) return hipErrorInvalidValue;
    else if (un.count) {
      hipLaunchKernelGGL((residual_bwd_kernel<T, TPR, V>), dim3((unsigned)un.count), dim3(TPR), 0, p.stream, p, un,
                         part_post, part_pre, part_gate);
    }
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  const unsigned cols = (p.K + 63) / 64;
  if (p.dg_post)
    hipLaunchKernelGGL(residual_reduce_kernel<float>, dim3(cols), dim3(1024), 0, p.stream, part_post, p.K, un.count,
                       p.dg_post, (int64_t)p.K);
  if (p.dg_pre)
    hipLaunchKernelGGL(residual_reduce_kernel<float>, dim3(cols), dim3(1024), 0, p.stream, part_pre, p.K, un.count,
                       p.dg_pre, (int64_t)p.K);
  if (part_gate)
    hipLaunchKernelGGL(residual_reduce_kernel<T>, dim3(cols, (unsigned)(un.count / un.pieces)), dim3(1024), 0, p.stream,
                       part_gate, p.K, (int64_t)un.pieces, (T*)p.dgate, (int64_t)p.lddg);
  return hipGetLastError();
}

}  // namespace

int64_t residual_bwd_ws_floats(int64_t M, int64_t K, int64_t gate_rows, int, bool post, bool pre, bool gate) {
  const Units un = units_of(M, gate_rows, gate);
  return un.count * K * ((post ? 1 : 0) + (pre ? 1 : 0) + (gate && un.pieces ? 1 : 0));
}

hipError_t launch_residual(const ResidualArgs& p) {
  return p.dtype == kDtypeBf16 ? launch_fwd_t<__bf16>(p) : launch_fwd_t<float>(p);
}

hipError_t launch_residual_bwd(const ResidualArgs& p) {
  return p.dtype == kDtypeBf16 ? launch_bwd_t<__bf16>(p) : launch_bwd_t<float>(p);
}

}  // namespace fn
