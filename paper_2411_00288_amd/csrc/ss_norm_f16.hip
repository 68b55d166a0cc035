// Norm kernels: SS_F16.
#include "ss_norm_kernel.h"

namespace ss {
SS_NORM_LAUNCHES(, SS_F16)
}
