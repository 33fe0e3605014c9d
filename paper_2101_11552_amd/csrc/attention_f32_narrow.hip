// The forward attention kernels for float32 heads of at most 32 columns.
#include "attention_launch.h"

namespace tfg {
TFG_ATTN_FWD(f32_narrow) { return launch_fwd_narrow<float>(p, s); }
}  // namespace tfg
