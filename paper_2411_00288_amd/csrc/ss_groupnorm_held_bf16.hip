// Group norm kernels that hold their data: SS_BF16.
#include "ss_groupnorm_held.h"

namespace ss {
SS_HELD_LAUNCHES(, SS_BF16)
}
