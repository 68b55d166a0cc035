// Group norm kernels: SS_BF16.
#include "ss_groupnorm_kernel.h"

namespace ss {
SS_GROUP_LAUNCHES(, SS_BF16)
}
