// Matrices held in 4 bits: launchers of the products with them, and what their kernels share.
#ifndef OZ2_W4_H
#define OZ2_W4_H

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/oz2.h"

// Launchers (oz2_w4.hip, oz2_w4_moe.hip); arguments as checked by the entry points.  alpha == 0 comes as an inner dimension of 0.
hipError_t oz2_launch_w4_matvec(const oz2_w4_matrix& w, int64_t t, float alpha, int x_type, const void* x, int64_t ldx, float beta,
                                const void* c, int64_t ldc, int y_type, void* y, int64_t ldy, hipStream_t st);
size_t oz2_w4_moe_space(const oz2_moe_layer& m, int64_t t);
hipError_t oz2_launch_w4_moe(const oz2_moe_layer& m, int64_t t, int x_type, const void* x, int64_t ldx, const uint8_t* active, int y_type,
                             void* y, int64_t ldy, int32_t* ids, float* weights, char* ws, hipStream_t st);

#ifdef __HIPCC__
__device__ __forceinline__ float w4_load(int type, const void* p, int64_t i) {
  if (type == OZ2_F32) return static_cast<const float*>(p)[i];
  if (type == OZ2_BF16) return __uint_as_float((unsigned)static_cast<const uint16_t*>(p)[i] << 16);
  return (float)static_cast<const _Float16*>(p)[i];
}

__device__ __forceinline__ void w4_store(int type, void* p, int64_t i, float v) {
  if (type == OZ2_F32) static_cast<float*>(p)[i] = v;
  else if (type == OZ2_BF16) static_cast<__bf16*>(p)[i] = (__bf16)v;
  else static_cast<_Float16*>(p)[i] = (_Float16)v;
}
#endif

#endif
