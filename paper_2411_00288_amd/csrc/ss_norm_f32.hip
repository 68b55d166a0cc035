// Norm kernels: SS_F32.
#include "ss_norm_kernel.h"

namespace ss {
SS_NORM_LAUNCHES(, SS_F32)
}
