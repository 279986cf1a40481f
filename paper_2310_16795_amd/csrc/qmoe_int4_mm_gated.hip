// k_int4_mm, gated, all zero points 8.
#include "qmoe_int4_mm.h"

namespace qmoe {

qmoe_status launch_int4_mm_gated(const Int4Args &a, int grid, hipStream_t s) { return launch_mm<true, false>(a, grid, s); }

}  // namespace qmoe
