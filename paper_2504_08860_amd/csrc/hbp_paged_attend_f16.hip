// Attention over a paged cache, all of it in fp16.
#include "hbp_paged_attend_rows.h"

namespace hbp {
int launch_attend_f16(const Attend &a, hipStream_t st) { return launch_attend<f16>(a, st); }
}  // namespace hbp
