// What the launch stubs of w4_stubs.cpp record (test infrastructure).
#pragma once
#include <hip/hip_runtime.h>

#include <vector>

#include "w4_kernels.h"

// A product's kernel: few rows (many = false) or many, the piece's rows and pointers, its workspace's parts.
struct stub_product {
  bool many;
  int epi, shape, M, NP, KB, splits;
  const void *a, *y;
  const float *inv_rms, *row_scale, *factor, *partial;
  int groups;
};
// Any other kernel.  The backward pass's partial sums are copied where stub_backward says that it is the kernel.
struct stub_launch {
  dim3 grid, block;
  const float* part[3];
};
extern std::vector<stub_product> stub_products;
extern std::vector<stub_launch> stub_launches;
extern bool stub_backward;

inline void stub_copy_args(stub_launch& l, void** args) {
  if (!stub_backward) return;
  for (int i = 0; i < 3; ++i) l.part[i] = *static_cast<const float**>(args[2 + i]);
}
