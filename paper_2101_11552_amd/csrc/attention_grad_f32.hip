// The attention's gradient kernels for float32 features.
#include "attention_grad.h"

namespace tfg {
int launch_grad_f32(AttnGrad& p, const RowPlan& r, hipStream_t s) { return launch_grad_type<float>(p, r, s); }
}  // namespace tfg
