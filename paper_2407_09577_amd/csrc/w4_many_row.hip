// Many-row kernels with 4-bit weights, EPI_ROWSCALE.
#include "w4_kernels.h"

namespace fn {
template hipError_t launch_w4_many<EPI_ROWSCALE>(const W4Gemm&, int, int, hipStream_t);
}
