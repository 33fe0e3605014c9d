// The attention's gradient kernels for bf16 features.
#include "attention_grad.h"

namespace tfg {
int launch_grad_bf16(AttnGrad& p, const RowPlan& r, hipStream_t s) { return launch_grad_type<__bf16>(p, r, s); }
}  // namespace tfg
