// Few-row kernels with 4-bit weights, EPI_RMS.
#include "w4_kernels.h"

namespace fn {
template hipError_t launch_w4_few<EPI_RMS>(const W4Args&, int);
}
