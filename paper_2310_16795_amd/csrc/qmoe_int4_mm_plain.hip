// k_int4_mm, one projection, all zero points 8.
#include "qmoe_int4_mm.h"

namespace qmoe {

qmoe_status launch_int4_mm_plain(const Int4Args &a, int grid, hipStream_t s) { return launch_mm<false, false>(a, grid, s); }

}  // namespace qmoe
