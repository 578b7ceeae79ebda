// oz2_attention in BF16 and FP16 with 129 to 256 values a head.  The sums of a wave, 128 registers, belong in accumulation registers here, so this file is compiled
// without -amdgpu-mfma-vgpr-form.
#include "oz2_attention_tile.h"

template <int XT>
hipError_t oz2_attention_wide_of(const Attention& a, hipStream_t st) {
  return oz2_attention_tile_launch<XT, 256, 4, 1>(a, st);
}
template hipError_t oz2_attention_wide_of<OZ2_BF16>(const Attention&, hipStream_t);
template hipError_t oz2_attention_wide_of<OZ2_F16>(const Attention&, hipStream_t);
