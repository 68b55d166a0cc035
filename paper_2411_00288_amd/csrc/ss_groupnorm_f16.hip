// Group norm kernels: SS_F16.
#include "ss_groupnorm_kernel.h"

namespace ss {
SS_GROUP_LAUNCHES(, SS_F16)
}
