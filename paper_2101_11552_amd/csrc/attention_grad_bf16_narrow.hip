// The attention's gradient kernels for bf16 heads of at most 32 columns.
#include "attention_grad_launch.h"

namespace tfg {
TFG_ATTN_GRAD(bf16_narrow) { return launch_grad_narrow<__bf16>(p, r, s); }
}  // namespace tfg
