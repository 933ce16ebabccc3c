// Few-row kernels with 4-bit weights, EPI_ROWSCALE.
#include "w4_kernels.h"

namespace fn {
template hipError_t launch_w4_few<EPI_ROWSCALE>(const W4Args&, int);
}
