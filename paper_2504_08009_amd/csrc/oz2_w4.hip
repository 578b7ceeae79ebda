// Products of a matrix held in 4 bits and a few vectors (oz2_w4_matvec).
#include "oz2_w4.h"

namespace {

// One wave a row and vector.
__global__ void __launch_bounds__(256) w4_matvec_kernel(oz2_w4_matrix w, float alpha, int x_type, const char* x, int64_t ldx, float beta,
                                                        const char* c, int64_t ldc, int y_type, char* y, int64_t ldy) {
  const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64, col = blockIdx.y;
  const int lane = threadIdx.x % 64;
  if (row >= w.n) return;
  const uint8_t* codes = static_cast<const uint8_t*>(w.codes) + row * w.ld_codes;
  float sum = 0.f;
  for (int64_t l = lane; l < w.k; l += 64) {
    const int q = codes[l / 2] >> (l % 2 * 4) & 15;
    const int64_t g = l / w.group;
    const int z = w.zeros ? static_cast<const uint8_t*>(w.zeros)[row * w.ld_zeros + g] : 8;
    sum = fmaf(w4_load(w.scale_type, w.scales, row * w.ld_scales + g) * (float)(q - z), w4_load(x_type, x, col * ldx + l), sum);
  }
  for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
  if (lane == 0) {
    float v = w.k ? alpha * sum : 0.f;
    if (beta != 0.f) v = fmaf(beta, w4_load(y_type, c, col * ldc + row), v);
    w4_store(y_type, y, col * ldy + row, v);
  }
}

}  // namespace

hipError_t oz2_launch_w4_matvec(const oz2_w4_matrix& w, int64_t t, float alpha, int x_type, const void* x, int64_t ldx, float beta,
                                const void* c, int64_t ldc, int y_type, void* y, int64_t ldy, hipStream_t st) {
  hipLaunchKernelGGL(w4_matvec_kernel, dim3((unsigned)((w.n + 3) / 4), (unsigned)t), dim3(256), 0, st, w, alpha, x_type,
                     static_cast<const char*>(x), ldx, beta, static_cast<const char*>(c), ldc, y_type, static_cast<char*>(y), ldy);
  return hipGetLastError();
}
