// The attention's gradient kernels for float32 heads of at most 32 columns.
#include "attention_grad_launch.h"

namespace tfg {
TFG_ATTN_GRAD(f32_narrow) { return launch_grad_narrow<float>(p, r, s); }
}  // namespace tfg
