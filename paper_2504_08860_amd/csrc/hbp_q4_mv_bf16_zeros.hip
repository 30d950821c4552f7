// Products with 4-bit matrices, x and y in bf16, with zero points.
#include "hbp_q4_mv_impl.h"

namespace hbp {
int launch_q4_mv_bf16_zeros(const Q4Product &p, hipStream_t st) { return launch_q4_mv<bf16, true>(p, st); }
}  // namespace hbp
