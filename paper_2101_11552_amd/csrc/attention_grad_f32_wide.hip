// The attention's gradient kernels for float32 heads of more than 32 columns.
#include "attention_grad_launch.h"

namespace tfg {
TFG_ATTN_GRAD(f32_wide) { return launch_grad_wide<float>(p, r, s); }
}  // namespace tfg
