// Attention over a paged cache, all of it in fp32.
#include "hbp_paged_attend_rows.h"

namespace hbp {
int launch_attend_f32(const Attend &a, hipStream_t st) { return launch_attend<float>(a, st); }
}  // namespace hbp
