// k_int4_mm, gated, with zero points.
#include "qmoe_int4_mm.h"

namespace qmoe {

qmoe_status launch_int4_mm_gated_zeros(const Int4Args &a, int grid, hipStream_t s) { return launch_mm<true, true>(a, grid, s); }

}  // namespace qmoe
