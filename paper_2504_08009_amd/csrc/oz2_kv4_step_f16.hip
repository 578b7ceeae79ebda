// oz2_kv4_attention with queries in F16.
#include "oz2_kv4_step.h"

template hipError_t oz2_kv4_step_of<OZ2_F16>(const Kv4Step&, dim3, hipStream_t);
