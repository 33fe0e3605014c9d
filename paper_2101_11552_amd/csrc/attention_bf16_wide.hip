// The forward attention kernels for bf16 heads of more than 32 columns.
#include "attention_launch.h"

namespace tfg {
TFG_ATTN_FWD(bf16_wide) { return launch_fwd_wide<__bf16>(p, s); }
}  // namespace tfg
