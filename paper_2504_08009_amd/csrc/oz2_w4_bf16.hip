// Products of a matrix held in 4 bits with vectors in BF16.
#include "oz2_w4_matvec.h"

template hipError_t oz2_w4_matvec_of<OZ2_BF16>(const W4Call&, int64_t);
