// First products of a layer of experts for tokens in F32.
#include "oz2_w4_moe_up.h"

template hipError_t oz2_moe_gate_up<OZ2_F32>(const MoeCall&, const oz2_w4_matrix&);
