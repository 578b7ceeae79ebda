// Products of a matrix held in 4 bits with vectors in F32.
#include "oz2_w4_matvec.h"

template hipError_t oz2_w4_matvec_of<OZ2_F32>(const W4Call&, int64_t);
