// Products with 4-bit matrices, x and y in bf16.
#include "hbp_q4_mv_impl.h"

namespace hbp {
int launch_q4_mv_bf16(const Q4Product &p, hipStream_t st) { return launch_q4_mv<bf16, false>(p, st); }
}  // namespace hbp
