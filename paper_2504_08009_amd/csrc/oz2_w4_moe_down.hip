// The experts' second products: part = weight (down h) for every place, summed over a token's places by a launch behind.
#include "oz2_w4_moe.h"
#ifndef MOE_DOWN_WAVES
#define MOE_DOWN_WAVES 3
#endif

namespace {

template <int T, int ST, bool ZEROS, int FOLD>
__global__ void __launch_bounds__(64 * kMoeWaves, T == 1 ? 4 : MOE_DOWN_WAVES) moe_down_kernel(MoeCall c, int split_log) {
  __shared__ Chosen chosen;
  __shared__ float part[2][kMoeRounds][kMoeWaves][4 * FOLD][T];
  const int n = c.chosen[0];
  if (threadIdx.x == 0) chosen.count = n;
  for (int i = threadIdx.x; i <= n; i += 64 * kMoeWaves) chosen.first[i] = c.chosen[1 + i];
  for (int i = threadIdx.x; i < n; i += 64 * kMoeWaves) chosen.expert[i] = c.chosen[2 + kMoePlaces + i];
  for (int i = threadIdx.x; i < c.t * c.top_k; i += 64 * kMoeWaves) chosen.place[i] = c.chosen[2 + 2 * kMoePlaces + i];
  __syncthreads();
  moe_products<OZ2_F32, T, ST, ZEROS, FOLD>(
      chosen, c.f, c.d, 4, split_log, c.down, part,
      [&](int64_t e) { return w4_of_stack(c.down, e, c.code_strides[2], c.scale_strides[2], c.zero_strides[2]); },
      [&](const W4Rows& m, int row, int i) { return w4_row<ST, FOLD>(m, row, i); },
      [&](int place) { return reinterpret_cast<const char*>(c.h + (int64_t)place * c.f); },
      [&](int place, int row, const float* u) {
        const float weight = c.weights[place];
#pragma unroll
        for (int i = 0; i < 4 * FOLD; ++i)
          if (row + i < c.d) c.part[(int64_t)place * c.d + row + i] = weight * u[i];
      });
}

__global__ void __launch_bounds__(256) moe_sum_kernel(MoeCall c) {
  const int i = blockIdx.x * 256 + threadIdx.x, t = blockIdx.y;
  if (i >= c.d) return;
  float v = 0.f;
  for (int j = 0; j < c.top_k; ++j) {
    const int place = t * c.top_k + j;
    if (c.ids[place] >= 0) v += c.part[(int64_t)place * c.d + i];
  }
  w4_store(c.y_type, c.y, t * c.ldy + i, v);
}

template <int T, int ST, bool ZEROS>
hipError_t launch_down(const MoeCall& c) {
  const dim3 grid(oz2_w4_compute_units() * (T == 1 ? 4 : MOE_DOWN_WAVES)), block(64 * kMoeWaves);
  if (moe_fold(c.down)) hipLaunchKernelGGL((moe_down_kernel<T, ST, ZEROS, 2>), grid, block, 0, c.st, c, 0);
  else hipLaunchKernelGGL((moe_down_kernel<T, ST, ZEROS, 1>), grid, block, 0, c.st, c, moe_split(c.f));
  hipLaunchKernelGGL(moe_sum_kernel, dim3((c.d + 255) / 256, c.t), dim3(256), 0, c.st, c);
  return hipGetLastError();
}
template <int T, int ST>
hipError_t launch_down(const MoeCall& c) {
  return c.down.zeros ? launch_down<T, ST, true>(c) : launch_down<T, ST, false>(c);
}

}  // namespace

hipError_t oz2_moe_down(const MoeCall& c, int scale_type) {
  if (!c.pairs) return scale_type == OZ2_F32 ? launch_down<1, OZ2_F32>(c) : scale_type == OZ2_BF16 ? launch_down<1, OZ2_BF16>(c) : launch_down<1, OZ2_F16>(c);
  return scale_type == OZ2_F32 ? launch_down<2, OZ2_F32>(c) : scale_type == OZ2_BF16 ? launch_down<2, OZ2_BF16>(c) : launch_down<2, OZ2_F16>(c);
}
