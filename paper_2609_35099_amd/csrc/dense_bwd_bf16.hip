// e3mi: the dense layers' backward in bfloat16.
#include "dense_bwd.h"

e3_status dense_bwd_bf16(const DenseBwdCall& c) { return dense_bwd_call<__bf16>(c); }
