// The forward attention kernels for bf16 heads of at most 32 columns.
#include "attention_launch.h"

namespace tfg {
TFG_ATTN_FWD(bf16_narrow) { return launch_fwd_narrow<__bf16>(p, s); }
}  // namespace tfg
