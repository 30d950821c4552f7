// Products with 4-bit matrices, x and y in fp32.
#include "hbp_q4_mv_impl.h"

namespace hbp {
int launch_q4_mv_f32(const Q4Product &p, hipStream_t st) { return launch_q4_mv<float, false>(p, st); }
}  // namespace hbp
