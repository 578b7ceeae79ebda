// oz2_attention in F16.
#include "oz2_attention_tile.h"

extern template hipError_t oz2_attention_wide_of<OZ2_F16>(const Attention&, hipStream_t);
template hipError_t oz2_attention_tile_of<OZ2_F16>(const Attention&, hipStream_t);
