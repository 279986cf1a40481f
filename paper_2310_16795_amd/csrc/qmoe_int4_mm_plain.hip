// k_int4_mm, one projection, all zero points 8.
#include "qmoe_int4_mm.h"

namespace qmoe {

qmoe_status launch_int4_mm_plain(const Int4Args &a, int cus, hipStream_t s) { return launch_mm<false, false>(a, cus, s); }

}  // namespace qmoe
