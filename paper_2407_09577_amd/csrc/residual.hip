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

// The sum over the first N = 2, 4, 8 or 16 lanes of each sixteen, where they repeat with that period, in every
// lane and in a fixed order.
template <int N>
__device__ __forceinline__ float lanes_total(float v) {
  auto add = [&](auto ctrl) __attribute__((always_inline)) {
    v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  add(std::integral_constant<int, 0xb1>{});                           // lanes 1, 0, 3, 2
  if constexpr (N >= 4) add(std::integral_constant<int, 0x4e>{});     // lanes 2, 3, 0, 1
  if constexpr (N >= 8) add(std::integral_constant<int, 0x141>{});    // 7 - i of eight
  if constexpr (N >= 16) add(std::integral_constant<int, 0x140>{});   // 15 - i of sixteen
  return v;
}

__device__ __forceinline__ float wave_total(float v) {
  v = lanes_total<16>(v);
  auto row = [&](int l) __attribute__((always_inline)) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l));
  };
  return (row(0) + row(16)) + (row(32) + row(48));
}

// Sums of NV values over the TPR threads of a row, the same in all of them and in a fixed order.  Several
// waves meet in LDS, in the two halves of buf by turns, so one barrier a call is enough: a wave writes a half
// again only after the barrier of the call between.
template <int TPR, int NV>
__device__ __forceinline__ void row_sum(float (&v)[NV], float (*buf)[NV][TPR / 64], int& turn) {
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = wave_total(v[i]);
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) buf[turn][i][threadIdx.x >> 6] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = lanes_total<TPR / 64>(buf[turn][i][threadIdx.x & (TPR / 64 - 1)]);
    turn ^= 1;
  }
}

// One workgroup of TPR threads per row, V vectors of 16 bytes per thread.  Bound by memory: 4096 x 4096 bf16 with a
// gate and both norms 28.2 us for 135 MB (4.8 TB/s), one row 2.1 us beside its launch.
template <typename T, int TPR, int V>
__global__ __launch_bounds__(TPR) void residual_kernel(ResidualArgs p) {
  constexpr int VN = Vec<T>::N;
  __shared__ float buf[2][1][TPR / 64];
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

// How the backward pass cuts the rows into units, each one workgroup's: ranges of rows that hold whole gate
// segments (pieces = 0: dgate is the unit's to write) or lie in one (pieces units per segment: dgate comes
// from their partial sums).  Without a gate, or with one per row, the rows are cut evenly.
struct Units {
  int64_t count;
  int rows, pieces;
};

// Enough units to fill the chip (eight waves per SIMD for narrow rows, four for wide), and no more: each
// leaves a row of fp32 partial sums per parameter.  A few rows are one unit, whose sums are the whole, so that no
// second launch adds them up (10 us in all for 2 to 16 rows of up to 4096): a row more takes 1.2 us with 64 threads
// (512 columns, 6 rows: 8.9 us), 2.1 with 512 (4096 columns, 3 rows: 8.8) and 7.6 with 1024 and two vectors each.
Units units_of(int64_t M, int64_t gate_rows, bool gate, int tpr) {
  const int64_t most = tpr <= 128 ? 2048 : tpr == 256 ? 1024 : 512;
  if (M == 0) return Units{0, 0, 0};
  if (M <= (tpr <= 128 ? 6 : tpr <= 512 ? 3 : 1)) return Units{1, (int)M, 0};
  int64_t rows = (M + most - 1) / most;
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
// in one pass over the row, after the first one (p).  The parameters' gradients add up in registers over the
// unit's rows.  Two workgroups of eight waves a compute unit hide each other's waits: with the next row's
// loads held ahead in registers only one fits (4096 x 4096 bf16, gate and both norms: 56 us, 43 without, for 229 MB).
// Rows of more than a vector a thread (more than 8192 bf16 or 4096 fp32 columns) are read three times: 3.1 TB/s of
// their bytes in bf16, 5.1 (4096 columns), 4.0 (8192) and 2.7 (16384) in fp32.
template <typename T, int TPR, int V, bool POST, bool PRE>
__global__ __launch_bounds__(TPR, TPR >= 512 ? 4 : 1) void residual_bwd_kernel(ResidualArgs p, Units un, float* part_post,
                                                                               float* part_pre, float* part_gate) {
  constexpr int VN = Vec<T>::N;
  __shared__ float buf1[2][1][TPR / 64];
  __shared__ float buf5[2][5][TPR / 64];
  int turn1 = 0, turn5 = 0;
  const int K = p.K;
  const float inv_k = 1.0f / (float)K;
  const int64_t u = blockIdx.x;
  int64_t m0, m1;
  if (un.pieces) {
    const int64_t s0 = u / un.pieces * p.gate_rows;
    m0 = s0 + u % un.pieces * un.rows;
    m1 = min(min(m0 + un.rows, s0 + (int64_t)p.gate_rows), (int64_t)p.M);
  } else {
    m0 = u * un.rows;
    m1 = min(m0 + un.rows, (int64_t)p.M);
  }
  // The sums over the unit's rows: in registers, but those of the norms' weights in LDS where a thread has
  // sixteen columns and no registers for them (each thread its own columns, so no barrier).
  constexpr bool kLds = V * VN >= 16;
  constexpr int VR = kLds ? 1 : V;
  __shared__ float lpost[kLds && POST ? V * VN : 1][kLds && POST ? TPR : 1];
  __shared__ float lpre[kLds && PRE ? V * VN : 1][kLds && PRE ? TPR : 1];
  float apost[VR][VN], apre[VR][VN], agate[V][VN];
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int e = 0; e < VN; ++e) {
      agate[j][e] = 0.0f;
      if constexpr (!kLds) apost[j][e] = apre[j][e] = 0.0f;
      if constexpr (kLds && POST) lpost[j * VN + e][threadIdx.x] = 0.0f;
      if constexpr (kLds && PRE) lpre[j * VN + e][threadIdx.x] = 0.0f;
    }
  // A thread's piece j of a row.  Lanes past K, and what a call has not, hold zeros (the gate: ones).
  struct Piece {
    Vec<T> x, h, gate, dho, dn;
    float gpost[VN], gpre[VN];
  };
  auto load_g = [&](int j, Piece& c) __attribute__((always_inline)) {
    const int k = (j * TPR + threadIdx.x) * VN;
#pragma unroll
    for (int e = 0; e < VN; ++e) c.gpost[e] = c.gpre[e] = 0.0f;
    if (k < K && POST) load_f32(p.g_post + k, c.gpost);
    if (k < K && PRE) load_f32(p.g_pre + k, c.gpre);
  };
  const u32x4 one = sizeof(T) == 2 ? u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u}
                                   : u32x4{0x3f800000u, 0x3f800000u, 0x3f800000u, 0x3f800000u};
  auto load = [&](int64_t m, int j, Piece& c) __attribute__((always_inline)) {
    const int k = (j * TPR + threadIdx.x) * VN;
    c.x.w = c.h.w = c.dho.w = c.dn.w = u32x4{0, 0, 0, 0};
    c.gate.w = one;
    if (k >= K) return;
    c.x.load((const T*)p.x + m * p.ldx + k);
    c.h.load((const T*)p.h + m * p.ldh + k);
    if (p.gate) c.gate.load((const T*)p.gate + m / p.gate_rows * p.ldg + k);
    if (p.dh_out) c.dho.load((const T*)p.dh_out + m * p.lddo + k);
    if constexpr (PRE) c.dn.load((const T*)p.dn + m * p.lddn + k);
  };
  // One piece a thread stays in registers over the row's three passes; with more each pass reads them again
  // (from the caches), as the three sums of every column leave no room to hold them.
  Piece c;
  if constexpr (V == 1) load_g(0, c);
  auto pass = [&](int64_t m, auto body) __attribute__((always_inline)) {
    if constexpr (V == 1) {
      body(0);
    } else {
      asm volatile("" ::: "memory");  // or the passes' equal loads become one, held in spilled registers
#pragma unroll
      for (int j = 0; j < V; ++j) {
        load_g(j, c);
        load(m, j, c);
        body(j);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  for (int64_t m = m0; m < m1; ++m) {
    if constexpr (V == 1) load(m, 0, c);
    float rp = 1.0f;
    if constexpr (POST) {
      float ss[1] = {0.f};
      pass(m, [&](int) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < VN; ++e) ss[0] = fmaf(c.x[e], c.x[e], ss[0]);
      });
      row_sum<TPR, 1>(ss, buf1, turn1);
      rp = rsqrtf(fmaf(ss[0], inv_k, p.eps_post));
    }
    float r = 0.f, t = 0.f, q = 0.f;
    auto scale = [&](int e) __attribute__((always_inline)) { return p.branch_scale * c.gate[e]; };
    auto branch = [&](int e) __attribute__((always_inline)) {  // v
      return (POST ? scale(e) * c.gpost[e] : scale(e)) * c.x[e];
    };
    auto H_of = [&](int e, float v) __attribute__((always_inline)) { return fmaf(v, rp, p.res_scale * c.h[e]); };
    if constexpr (POST || PRE) {
      float s5[5] = {0.f, 0.f, 0.f, 0.f, 0.f};  // H^2, a H, v dH, v a, v H
      pass(m, [&](int) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < VN; ++e) {
          const float v = branch(e);
          if constexpr (PRE) {
            const float H = H_of(e, v), a = c.dn[e] * c.gpre[e];
            s5[0] = fmaf(H, H, s5[0]);
            s5[1] = fmaf(a, H, s5[1]);
            s5[3] = fmaf(v, a, s5[3]);
            s5[4] = fmaf(v, H, s5[4]);
          }
          s5[2] = fmaf(v, c.dho[e], s5[2]);
        }
      });
      row_sum<TPR, 5>(s5, buf5, turn5);
      if constexpr (PRE) {
        r = rsqrtf(fmaf(s5[0], inv_k, p.eps_pre));
        t = r * s5[1] * inv_k;
      }
      q = rp * (s5[2] + r * (s5[3] - r * t * s5[4])) * inv_k;
    }
    pass(m, [&](int j) __attribute__((always_inline)) {
      const int k = (j * TPR + threadIdx.x) * VN;
      float odx[VN], odh[VN];
#pragma unroll
      for (int e = 0; e < VN; ++e) {
        float D = c.dho[e];
        if constexpr (PRE) {
          const float Hr = H_of(e, branch(e)) * r;
          D = fmaf(r, fmaf(-Hr, t, c.dn[e] * c.gpre[e]), D);
          if constexpr (kLds) lpre[j * VN + e][threadIdx.x] = fmaf(c.dn[e], Hr, lpre[j * VN + e][threadIdx.x]);
          else apre[j][e] = fmaf(c.dn[e], Hr, apre[j][e]);
        }
        const float xp = c.x[e] * rp, dz = scale(e) * D, Dx = D * xp;
        odh[e] = p.res_scale * D;
        odx[e] = POST ? rp * fmaf(-xp, q, dz * c.gpost[e]) : dz;
        agate[j][e] = fmaf(POST ? Dx * c.gpost[e] : Dx, p.branch_scale, agate[j][e]);
        if constexpr (POST && kLds) lpost[j * VN + e][threadIdx.x] = fmaf(dz, xp, lpost[j * VN + e][threadIdx.x]);
        else if constexpr (POST) apost[j][e] = fmaf(dz, xp, apost[j][e]);
      }
      if (k < K) {
        store_vec<T>((T*)p.dx + m * p.lddx + k, odx);
        store_vec<T>((T*)p.dh + m * p.lddh + k, odh);
      }
    });
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
  auto keep = [&](float* part, auto value) __attribute__((always_inline)) {
    if (!part) return;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int k = (j * TPR + threadIdx.x) * VN;
      if (k >= K) continue;
#pragma unroll
      for (int i = 0; i < VN; i += 4)
        *reinterpret_cast<f32x4*>(part + u * K + k + i) =
            f32x4{value(j, i), value(j, i + 1), value(j, i + 2), value(j, i + 3)};
    }
  };
  if constexpr (POST)
    keep(part_post, [&](int j, int e) {
      if constexpr (kLds) return lpost[j * VN + e][threadIdx.x];
      else return apost[j][e];
    });
  if constexpr (PRE)
    keep(part_pre, [&](int j, int e) {
      if constexpr (kLds) return lpre[j * VN + e][threadIdx.x];
      else return apre[j][e];
    });
  keep(part_gate, [&](int j, int e) { return agate[j][e]; });
}

// Sums of the units' partials in a fixed order.  A workgroup takes 32 columns of one sum (blockIdx.y: dg_post,
// dg_pre, then the gate's segments, as far as the call has them): eight threads read 128 bytes of a partial
// row, 32 rows at a time.  512 units of 4096 columns: 6.4 us for 25 MB, most of it latency.
template <typename T>
__global__ __launch_bounds__(256) void residual_sums_kernel(ResidualArgs p, Units un, const float* part_post,
                                                            const float* part_pre, const float* part_gate) {
  __shared__ f32x4 red[32][8];
  const int q = threadIdx.x & 7, w = threadIdx.x >> 3, k = (blockIdx.x * 8 + q) * 4, K = p.K;
  int which = blockIdx.y;
  const float* part = nullptr;
  float* out = nullptr;
  int64_t count = un.count;
  if (p.dg_post && which-- == 0) part = part_post, out = p.dg_post;
  else if (p.dg_pre && which-- == 0) part = part_pre, out = p.dg_pre;
  else part = part_gate + (int64_t)which * un.pieces * K, count = un.pieces;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (k < K) {
    for (int64_t u0 = w; u0 < count; u0 += 32 * 8) {
      f32x4 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (u0 + 32 * i < count) v[i] = *reinterpret_cast<const f32x4*>(part + (u0 + 32 * i) * K + k);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
    }
  }
  red[w][q] = s;
  __syncthreads();
  if (w || k >= K) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) s += red[i][q];
  if (out) {
    *reinterpret_cast<f32x4*>(out + k) = s;
  } else if constexpr (sizeof(T) == 2) {
    const float o[4] = {s[0], s[1], s[2], s[3]};
    *reinterpret_cast<u32x2*>((T*)p.dgate + (int64_t)which * p.lddg + k) = pack4_bf16(o);
  } else {
    *reinterpret_cast<f32x4*>((T*)p.dgate + (int64_t)which * p.lddg + k) = s;
  }
}

// Threads per row and vectors per thread: the fewest threads that hold the row's n vectors of 16 bytes one
// apiece; 1024 threads with two or four beyond.
int threads_of(int64_t K, int dtype) {
  const int64_t n = K / (dtype == kDtypeBf16 ? 8 : 4);
  return n <= 64 ? 64 : n <= 128 ? 128 : n <= 256 ? 256 : n <= 512 ? 512 : 1024;
}

template <typename T, typename F>
hipError_t with_shape(int K, F go) {
  const int n = K / Vec<T>::N;
  if (n <= 64) return go(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  if (n <= 128) return go(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{});
  if (n <= 256) return go(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
  if (n <= 512) return go(std::integral_constant<int, 512>{}, std::integral_constant<int, 1>{});
  if (n <= 1024) return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
  if (n <= 2048) return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
  if constexpr (sizeof(T) == 4) return go(std::integral_constant<int, 1024>{}, std::integral_constant<int, 4>{});
  return hipErrorInvalidValue;
}

template <typename T>
hipError_t launch_fwd_t(const ResidualArgs& p) {
  return with_shape<T>(p.K, [&](auto tpr, auto v) {
    constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value;
    hipLaunchKernelGGL((residual_kernel<T, TPR, V>), dim3(min(p.M, 1 << 20)), dim3(TPR), 0, p.stream, p);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t launch_bwd_t(const ResidualArgs& p) {
  const Units un = units_of(p.M, p.gate_rows, p.dgate != nullptr, threads_of(p.K, p.dtype));
  float* next = p.ws;
  auto take = [&](bool wanted) {
    float* q = wanted ? next : nullptr;
    if (wanted) next += un.count * p.K;
    return q;
  };
  float* part_post = un.count == 1 ? p.dg_post : take(p.dg_post != nullptr);
  float* part_pre = un.count == 1 ? p.dg_pre : take(p.dg_pre != nullptr);
  float* part_gate = take(p.dgate && un.pieces);
  if (un.count) {
    const hipError_t e = with_shape<T>(p.K, [&](auto tpr, auto v) {
      constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value;
      auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)un.count), dim3(TPR), 0, p.stream, p, un, part_post, part_pre, part_gate);
        return hipGetLastError();
      };
      if (p.g_post) return p.g_pre ? go(residual_bwd_kernel<T, TPR, V, true, true>) : go(residual_bwd_kernel<T, TPR, V, true, false>);
      return p.g_pre ? go(residual_bwd_kernel<T, TPR, V, false, true>) : go(residual_bwd_kernel<T, TPR, V, false, false>);
    });
    if (e != hipSuccess) return e;
  }
  if (un.count == 1) return hipSuccess;
  const unsigned sums = (p.dg_post ? 1 : 0) + (p.dg_pre ? 1 : 0) + (part_gate ? (unsigned)(un.count / un.pieces) : 0);
  if (!sums) return hipSuccess;
  hipLaunchKernelGGL(residual_sums_kernel<T>, dim3((p.K + 31) / 32, sums), dim3(256), 0, p.stream, p, un, part_post, part_pre,
                     part_gate);
  return hipGetLastError();
}

}  // namespace

int64_t residual_bwd_ws_floats(int64_t M, int64_t K, int64_t gate_rows, int dtype, bool post, bool pre, bool gate) {
  const Units un = units_of(M, gate_rows, gate, threads_of(K, dtype));
  return un.count * K * ((post ? 1 : 0) + (pre ? 1 : 0) + (gate && un.pieces ? 1 : 0));
}

hipError_t launch_residual(const ResidualArgs& p) {
  return p.dtype == kDtypeBf16 ? launch_fwd_t<__bf16>(p) : launch_fwd_t<float>(p);
}

hipError_t launch_residual_bwd(const ResidualArgs& p) {
  return p.dtype == kDtypeBf16 ? launch_bwd_t<__bf16>(p) : launch_bwd_t<float>(p);
}

}  // namespace fn
