// The forward attention kernels for float32 features.
#include "attention_fwd.h"

namespace tfg {
int launch_fwd_f32(AttnFwd& p, hipStream_t s) { return launch_fwd_type<float>(p, s); }
}  // namespace tfg
