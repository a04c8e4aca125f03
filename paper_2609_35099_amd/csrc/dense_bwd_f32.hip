// e3mi: the dense layers' backward in float32.
#include "dense_bwd.h"

e3_status dense_bwd_f32(const DenseBwdCall& c) { return dense_bwd_call<float>(c); }
