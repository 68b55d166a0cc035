// Group norm kernels that hold their data: SS_F32.
#include "ss_groupnorm_held.h"

namespace ss {
SS_HELD_LAUNCHES(, SS_F32)
}
