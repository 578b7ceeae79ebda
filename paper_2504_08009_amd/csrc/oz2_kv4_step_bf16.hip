// oz2_kv4_attention with queries in BF16.
#include "oz2_kv4_step.h"

template hipError_t oz2_kv4_step_of<OZ2_BF16>(const Kv4Step&, dim3, hipStream_t);
