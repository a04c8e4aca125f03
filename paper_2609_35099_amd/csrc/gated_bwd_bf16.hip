// e3mi: the narrow gated layers' backward in bfloat16.
#include "gated_bwd.h"

e3_status gated_bwd_fused_bf16(const GatedCall& c) { return gated_bwd_fused<__bf16>(c); }
