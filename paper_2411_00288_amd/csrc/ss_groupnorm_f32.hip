// Group norm kernels: SS_F32.
#include "ss_groupnorm_kernel.h"

namespace ss {
SS_GROUP_LAUNCHES(, SS_F32)
}
