// k_int4_mm, one projection, with zero points.
#include "qmoe_int4_mm.h"

namespace qmoe {

qmoe_status launch_int4_mm_zeros(const Int4Args &a, int grid, hipStream_t s) { return launch_mm<false, true>(a, grid, s); }

}  // namespace qmoe
