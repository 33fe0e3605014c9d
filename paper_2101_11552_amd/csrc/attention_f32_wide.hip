// The forward attention kernels for float32 heads of more than 32 columns.
#include "attention_launch.h"

namespace tfg {
TFG_ATTN_FWD(f32_wide) { return launch_fwd_wide<float>(p, s); }
}  // namespace tfg
