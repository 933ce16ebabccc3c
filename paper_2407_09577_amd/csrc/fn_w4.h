// 4-bit weights: the packed layout, shared by the folds and the products.
//
// A weight is held as codes q = 0..15 with, for each group of G = 32, 64 or 128 consecutive k of a
// column, a scale s and a zero point z = 0..63: it stands for (q - z) s.  Packed columns are those
// of fn_device.h (a GLU pairs gate and up blocks), padded to NP (a multiple of 16), and K is padded
// to a multiple of 128.  The buffer holds
//   codes   fragments of 1 KiB, k-block major: fragment (kb, cb) = 128 rows k x 16 columns at byte
//           (kb * NP/16 + cb) * 1024; lane L = 16 c + p holds 16 bytes, word u the eight k =
//           128 kb + 32 u + 8 c + e of column 16 cb + p: the operand of four matrix-core steps, so
//           a wave loads a fragment with one 16-byte access per lane;
//   scales  after the codes, one 32-bit word per group and packed column, [groups][NP] (groups of
//           the padded K): the fp32 s rounded to 12 significant bits, which hold every bf16 and
//           fp16 value, with z in the low six.
//   norms   after the scales, an fp32 power of two per packed column, [NP]: what brings the column's
//           largest |s| into [2^9, 2^10), for the many-row kernel's fp16 weights.
// Code e of a word is the nibble at bit 4 (e / 2) + 16 (e % 2): (word >> 4 i) & 0x000f000f are the
// codes 2 i and 2 i + 1 in the halves of a register, and one and-or makes two weights of them.
//
// Few rows: OR'ed with 0x4300 a half is the bf16 128 + q, exactly, and the group's sum of the
// activations takes the 128 + z off again:
//   sum_k a (q - z) s = s (sum_k a (128 + q) - (128 + z) sum_k a).
// No weight is rounded: the bf16 products are exact, the sums are fp32.  The offset costs last bits of
// them: partial sums below 143 sum |a| and, with z up to 63, 191 sum |a| leave a group off by at most 2^-10
// of |s| sum |a|, whatever its codes (a group that stands for zeros has that residue too).  For codes
// spread around z it is some 2^-18 of sum |a w|.
// Many rows: OR'ed with 0x6400 a half is the fp16 1024 + q; less 1024 + z, times the scale as fp16, it is
// the weight in eleven bits (w4_kernels.h).
// The products run with the activations as the matrix cores' first operand, so a lane's four results
// are four rows of one column, whose scale word is the one that its codes need too.
#pragma once

#include "fn_device.h"

namespace fn {

constexpr int kW4KB = 128;         // k extent of a code fragment
constexpr float kW4Bias = 128.0f;  // added to every code by its bf16 form
constexpr unsigned kW4ScaleMask = 0xfffff000u;

// Between a wave's writes to LDS and its lanes' reads of what others of its lanes wrote, and before it writes there again:
// a wave's accesses to LDS are done in the order in which they are issued, and past this no memory access is moved by the
// compiler, which otherwise keeps that order only as long as it cannot tell the addresses apart.  No instruction comes of
// it.
__device__ __forceinline__ void wave_lds_order() { __builtin_amdgcn_wave_barrier(); }

// Bit of code e (0..7) in its word.
__device__ __forceinline__ constexpr int w4_bit(int e) { return 4 * (e >> 1) + 16 * (e & 1); }

// The and-or's operands in registers, a scalar and a vector one: with literals, which it cannot take, it becomes two
// instructions, and the widening is what the products' vector units do most (the few-row kernel at 64 x 11008 -> 4096:
// 18.6 us with literals, 17.7 so).
struct W4Bits {
  unsigned low, high, bias;
  __device__ __forceinline__ explicit W4Bits(unsigned b) : low(0x000f000fu), high(0x00f000f0u), bias(b) {
    asm("" : "+s"(low));
    asm("" : "+s"(high));
    asm("" : "+v"(bias));
  }
};

// The eight codes of a word as bf16 128 + q, in k order (the bias: 0x43004300).
__device__ __forceinline__ bf16x8 w4_widen(unsigned w, const W4Bits& k) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = ((w >> (4 * i)) & k.low) | k.bias;
  return __builtin_bit_cast(bf16x8, r);
}

__device__ __forceinline__ float w4_scale(unsigned word) { return __uint_as_float(word & kW4ScaleMask); }
__device__ __forceinline__ float w4_zero(unsigned word) { return (float)(word & 63u); }

}  // namespace fn
