// Launch stubs for the host-only sanitizer build of the 4-bit products, the folds and the block residual (test
// infrastructure): the launchers of the real sources run; the product kernels' launchers and the HIP runtime entry
// points below them record what they are given, so a machine without a GPU can check it.
#include "w4_stub_record.h"

#include <hip/hip_runtime.h>

std::vector<stub_product> stub_products;
std::vector<stub_launch> stub_launches;

namespace fn {
#define FEW(EPI)                                                                                             \
  template <>                                                                                                \
  hipError_t launch_w4_few<EPI>(const W4Args& p, int shape) {                                                \
    stub_products.push_back(stub_product{false, EPI, shape, p.M, p.NP, p.KB, 1, p.a, p.y, p.ep.inv_rms, p.ep.row_scale, \
                                         nullptr, nullptr, 0});                                              \
    return hipSuccess;                                                                                       \
  }                                                                                                          \
  template <>                                                                                                \
  hipError_t launch_w4_many<EPI>(const W4Gemm& q, int, int shape, hipStream_t) {                             \
    stub_products.push_back(stub_product{true, EPI, shape, q.M, q.NP, q.KB, q.splits, q.a, q.y, nullptr, q.row_scale, q.factor, \
                                         q.partial, q.groups});                                              \
    return hipSuccess;                                                                                       \
  }
FEW(EPI_RMS)
FEW(EPI_GLU)
FEW(EPI_ROWSCALE)
}  // namespace fn

namespace {
stub_launch next;
}

extern "C" {
void** __hipRegisterFatBinary(const void*) {
  static void* h;
  return &h;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterVar(void*, void*, char*, const char*, int, unsigned long, int, int) {}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, void*, void*, int*) {}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  next = stub_launch{grid, block, {}};
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* stream) {
  *grid = next.grid, *block = next.block, *shared = 0, *stream = nullptr;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void*, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
  next = stub_launch{grid, block, {}};
  stub_copy_args(next, args);
  stub_launches.push_back(next);
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
}
