// Products with 4-bit matrices, x and y in fp32, with zero points.
#include "hbp_q4_mv_impl.h"

namespace hbp {
int launch_q4_mv_f32_zeros(const Q4Product &p, hipStream_t st) { return launch_q4_mv<float, true>(p, st); }
}  // namespace hbp
