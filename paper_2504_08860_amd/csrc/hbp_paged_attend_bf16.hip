// Attention over a paged cache, all of it in bf16.
#include "hbp_paged_attend_rows.h"

namespace hbp {
int launch_attend_bf16(const Attend &a, hipStream_t st) { return launch_attend<bf16>(a, st); }
}  // namespace hbp
