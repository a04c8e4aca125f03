// e3mi: the gated layers' forward in float32.
#include "gated.h"

e3_status gated_fwd_f32(const GatedCall& c) { return gated_fwd<float>(c); }
