// e3mi: the narrow gated layers' backward in float32.
#include "gated_bwd.h"

e3_status gated_bwd_fused_f32(const GatedCall& c) { return gated_bwd_fused<float>(c); }
