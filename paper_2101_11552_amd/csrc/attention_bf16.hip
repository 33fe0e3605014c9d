// The forward attention kernels for bf16 features.
#include "attention_fwd.h"

namespace tfg {
int launch_fwd_bf16(AttnFwd& p, hipStream_t s) { return launch_fwd_type<__bf16>(p, s); }
}  // namespace tfg
