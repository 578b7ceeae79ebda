// Products of a matrix held in 4 bits and a few vectors (oz2_w4_matvec): dispatch by the type of the vectors.
#include "oz2_w4_matvec.h"

extern template hipError_t oz2_w4_matvec_of<OZ2_F32>(const W4Call&, int64_t);
extern template hipError_t oz2_w4_matvec_of<OZ2_BF16>(const W4Call&, int64_t);
extern template hipError_t oz2_w4_matvec_of<OZ2_F16>(const W4Call&, int64_t);

namespace {

// What the loads of the other kernels do not fit: rows of a few bytes, or further apart than they count.  One wave a row and vector, and the rows a grid
// behind it: a launch has fewer than 2^32 threads in a dimension, a matrix up to 2^31 rows.
constexpr int64_t kSimpleGroups = 1 << 22;
__global__ void __launch_bounds__(256) w4_simple_kernel(oz2_w4_matrix w, float alpha, int x_type, const char* x, int64_t ldx, float beta,
                                                        const char* c, int64_t ldc, int y_type, char* y, int64_t ldy) {
  const int64_t col = blockIdx.y;
  const int lane = threadIdx.x % 64;
  for (int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64; row < w.n; row += (int64_t)gridDim.x * 4) {
    const uint8_t* codes = static_cast<const uint8_t*>(w.codes) + row * w.ld_codes;
    float sum = 0.f;
    for (int64_t l = lane; l < w.k; l += 64) {
      const int q = codes[l / 2] >> (l % 2 * 4) & 15;
      const int64_t g = l / w.group;
      const int z = w.zeros ? static_cast<const uint8_t*>(w.zeros)[row * w.ld_zeros + g] : 8;
      sum = fmaf(w4_load(w.scale_type, w.scales, row * w.ld_scales + g) * (float)(q - z), w4_load(x_type, x, col * ldx + l), sum);
    }
    for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
    if (lane) continue;
    float v = w.k ? alpha * sum : 0.f;
    if (beta != 0.f) v = fmaf(beta, w4_load(y_type, c, col * ldc + row), v);
    w4_store(y_type, y, col * ldy + row, v);
  }
}

}  // namespace

W4Rows oz2_w4_rows(const oz2_w4_matrix& m) {
  W4Rows w;
  w.codes = static_cast<const uint8_t*>(m.codes);
  w.scales = static_cast<const char*>(m.scales);
  w.zeros = static_cast<const uint8_t*>(m.zeros);
  w.ld_codes = m.ld_codes, w.ld_scales = m.ld_scales, w.ld_zeros = m.ld_zeros;
  w.n = (int)m.n, w.k = (int)m.k;
  w.group = (int)(m.group < ((int64_t)1 << 23) ? m.group : (int64_t)1 << 23);  // (k is below that)
  w.bytes = (w.k + 1) / 2;
  w.full = w.k / kW4Block;
  w.groups = (int)((m.k + m.group - 1) / m.group);
  const int64_t per = m.group / kW4Block, blocks = w.full + 1;
  const int64_t of_group = per < blocks ? per : blocks;
  w.recip = of_group <= 1 ? 0u : (unsigned)((((int64_t)1 << 32) + of_group - 1) / of_group);
  w.keep = of_group <= 1 ? ~0u : 0u;
  return w;
}

hipError_t oz2_launch_w4_matvec(const oz2_w4_matrix& m, int64_t t, float alpha, int x_type, const void* x, int64_t ldx, float beta,
                                const void* c, int64_t ldc, int y_type, void* y, int64_t ldy, hipStream_t st) {
  const W4Call a = {oz2_w4_rows(m), m.scale_type, (int)t, alpha, beta, x, c, ldx, ldc, ldy, y_type, y, st};
  if (m.k < 32 || !w4_tile_fits(a.w)) {
    const int64_t groups = (m.n + 3) / 4;
    hipLaunchKernelGGL(w4_simple_kernel, dim3((unsigned)(groups < kSimpleGroups ? groups : kSimpleGroups), (unsigned)t), dim3(256), 0, st, m, alpha, x_type,
                       static_cast<const char*>(x), ldx, beta, static_cast<const char*>(c), ldc, y_type, static_cast<char*>(y), ldy);
    return hipGetLastError();
  }
  return x_type == OZ2_F32    ? oz2_w4_matvec_of<OZ2_F32>(a, m.group)
         : x_type == OZ2_BF16 ? oz2_w4_matvec_of<OZ2_BF16>(a, m.group)
                              : oz2_w4_matvec_of<OZ2_F16>(a, m.group);
}
