// e3mi: the gated layers' forward in bfloat16.
#include "gated.h"

e3_status gated_fwd_bf16(const GatedCall& c) { return gated_fwd<__bf16>(c); }
