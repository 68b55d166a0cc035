// Norm kernels: SS_BF16.
#include "ss_norm_kernel.h"

namespace ss {
SS_NORM_LAUNCHES(, SS_BF16)
}
