// The attention's gradient kernels for bf16 heads of more than 32 columns.
#include "attention_grad_launch.h"

namespace tfg {
TFG_ATTN_GRAD(bf16_wide) { return launch_grad_wide<__bf16>(p, r, s); }
}  // namespace tfg
