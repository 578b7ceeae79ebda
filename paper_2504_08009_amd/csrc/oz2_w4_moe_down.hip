// The experts' second products: part = weight (down h) for every place, summed over a token's places by a launch behind.
#include "oz2_w4_moe.h"

namespace {

// What the launch before has left of its choice.
__device__ __forceinline__ void moe_chosen(const MoeCall& c, Chosen& chosen) {
  const int n = c.chosen[0];
  if (threadIdx.x == 0) chosen.count = n;
  for (int i = threadIdx.x; i <= n; i += 64 * kMoeWaves) chosen.first[i] = c.chosen[1 + i];
  for (int i = threadIdx.x; i < n; i += 64 * kMoeWaves) chosen.expert[i] = c.chosen[2 + kMoePlaces + i];
  for (int i = threadIdx.x; i < c.t * c.top_k; i += 64 * kMoeWaves) chosen.place[i] = c.chosen[2 + 2 * kMoePlaces + i];
  __syncthreads();
}
__device__ __forceinline__ W4Rows moe_down_of(const MoeCall& c, int64_t e) {
  return w4_of_stack(c.down, e, c.code_strides[2], c.scale_strides[2], c.zero_strides[2]);
}

template <int ST, bool ZEROS, int FOLD>
__global__ void __launch_bounds__(64 * kMoeWaves, 4) moe_down_kernel(MoeCall c, int split_log) {
  __shared__ Chosen chosen;
  __shared__ float part[2][kMoeRounds][kMoeWaves][4 * FOLD];
  moe_chosen(c, chosen);
  moe_products<OZ2_F32, ST, ZEROS, FOLD>(
      chosen, c.f, c.d, 4, split_log, c.down, part, [&](int64_t e) { return moe_down_of(c, e); },
      [&](const W4Rows& m, int row, int i) { return w4_row<ST, FOLD>(m, row, i); },
      [&](int place) { return reinterpret_cast<const char*>(c.h + (int64_t)place * c.f); },
      [&](int place, int row, const float* u) {
        const float weight = c.weights[place];
#pragma unroll
        for (int i = 0; i < 4 * FOLD; ++i)
          if (row + i < c.d) c.part[(int64_t)place * c.d + row + i] = weight * u[i];
      });
}

// BATCHES batches of rows for all places of a token, and their sums.  Groups of `1 << split_log` waves take every per-th place each: eight waves, so that
// most tokens' places are all in flight.  A lane brings 128 bytes of h for the 64 of codes in a batch's four loads: two batches where there are still four
// workgroups a compute unit: 4 tokens through 6 of 64 experts of 4096 x 1024 in half precision 60 -> 55 us, 8 through 4 of 128 of 2048 x 2048 85 -> 75.
// (With zero points and two rows a load the compiler keeps 48 bytes a lane of it in scratch memory.)
constexpr int kDirectWaves = 8;
template <int ST, bool ZEROS, int FOLD, int BATCHES>
__global__ void __launch_bounds__(64 * kDirectWaves, 4) moe_down_direct_kernel(MoeCall c, int split_log) {
  constexpr int ROWS = 4 * FOLD;
  __shared__ float part[kDirectWaves][BATCHES * ROWS];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, token = blockIdx.y;
  const int split = 1 << split_log, group = wave >> split_log, per = kDirectWaves >> split_log;
  const int unit = FOLD == 2 ? lane % 32 : (wave & (split - 1)) * 64 + lane, row = blockIdx.x * BATCHES * ROWS;
  const W4Place at = w4_place(c.down, unit);
  const bool ragged = __ballot(at.cut != 0) != 0;
  float mine[BATCHES][FOLD];
#pragma unroll
  for (int i = 0; i < BATCHES * FOLD; ++i) mine[i / FOLD][i % FOLD] = 0.f;
  for (int j = group; j < c.top_k; j += per) {
    const int place = token * c.top_k + j, e = __builtin_amdgcn_readfirstlane(c.ids[place]);
    if (e < 0) break;  // (and so are those behind)
    const float weight = c.weights[place];
    const W4Rows m = moe_down_of(c, e);
    auto vector = [&](int) { return reinterpret_cast<const char*>(c.h + (int64_t)place * c.f); };
    W4Rows4<OZ2_F32, 1, ST, ZEROS, FOLD> r[BATCHES];
    w4_each<BATCHES>([&](auto b) __attribute__((always_inline)) { r[b.value].fetch([&](int i) { return w4_row<ST, FOLD>(m, row + b.value * ROWS, i); }, at); });
    W4X<OZ2_F32> kept[1];
    const unsigned plain = w4_take_x<OZ2_F32, 1>(c.f, unit, vector, kept);
    w4_each<BATCHES>([&](auto b) __attribute__((always_inline)) {
      float sum[4][1], v[FOLD];
      r[b.value].multiply(at, kept, ragged, sum);
      if (plain) r[b.value].multiply_plain(plain, c.f, c.down.group, [&](int i) { return w4_row<ST, FOLD>(m, row + b.value * ROWS, i); }, vector, unit, sum);
      w4_sum4<FOLD>(sum[0][0], sum[1][0], sum[2][0], sum[3][0], v);
#pragma unroll
      for (int i = 0; i < FOLD; ++i) mine[b.value][i] = fmaf(weight, v[i], mine[b.value][i]);
    });
  }
  if (lane % 16 == 0)
#pragma unroll
    for (int i = 0; i < BATCHES * FOLD; ++i) part[wave][i / FOLD * ROWS + w4_row_of_lane<FOLD>(i % FOLD)] = mine[i / FOLD][i % FOLD];
  __syncthreads();
  if (threadIdx.x >= BATCHES * ROWS || row + (int)threadIdx.x >= c.d) return;
  float v = 0.f;
#pragma unroll
  for (int q = 0; q < kDirectWaves; ++q) v += part[q][threadIdx.x];
  w4_store(c.y_type, c.y, token * c.ldy + row + threadIdx.x, v);
}

template <int SPB, int RT, bool WIDE, bool ZEROS>
__global__ void __launch_bounds__(64 * kMoeWaves, kMoeFit) moe_down_tiles_kernel(MoeCall c, int scale_type) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ Chosen chosen;
  moe_chosen(c, chosen);
  moe_tiles<OZ2_F32, SPB, RT, WIDE, ZEROS>(
      chosen, c.t, c.f, c.d, 32, scale_type, lds, [&](int64_t e) { return moe_down_of(c, e); }, [](const W4Rows& m, int) { return m; },
      [](int row, int t) { return row + 16 * t; }, [&](int place) { return reinterpret_cast<const char*>(c.h + (int64_t)place * c.f); },
      [&](int place, int row, float u0, float u1) {
        const float weight = c.weights[place];
        if (row < c.d) c.part[(int64_t)place * c.d + row] = weight * u0;
        if (row + 16 < c.d) c.part[(int64_t)place * c.d + row + 16] = weight * u1;
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

template <int ST, bool ZEROS, int FOLD, int BATCHES>
void launch_direct(const MoeCall& c, int split) {
  constexpr int rows = BATCHES * 4 * FOLD;
  hipLaunchKernelGGL((moe_down_direct_kernel<ST, ZEROS, FOLD, BATCHES>), dim3((c.d + rows - 1) / rows, c.t), dim3(64 * kDirectWaves), 0, c.st, c, split);
}
template <int ST, bool ZEROS, int FOLD>
void launch_down(const MoeCall& c, int split) {
  if (!c.direct) hipLaunchKernelGGL((moe_down_kernel<ST, ZEROS, FOLD>), dim3(oz2_w4_compute_units() * 4), dim3(64 * kMoeWaves), 0, c.st, c, split);
  else if ((int64_t)c.d * c.t < (int64_t)oz2_w4_compute_units() * 4 * 8 * FOLD) launch_direct<ST, ZEROS, FOLD, 1>(c, split);
  else launch_direct<ST, ZEROS, FOLD, 2>(c, split);
}
template <int ST, bool ZEROS>
void launch_down(const MoeCall& c) {
  if (moe_fold(c.down)) launch_down<ST, ZEROS, 2>(c, 0);
  else launch_down<ST, ZEROS, 1>(c, moe_split(c.f));
}
template <int ST>
void launch_down(const MoeCall& c) {
  c.down.zeros ? launch_down<ST, true>(c) : launch_down<ST, false>(c);
}
template <int SPB, int RT, bool WIDE, bool ZEROS>
void launch_down_tiles(const MoeCall& c, int scale_type) {
  hipLaunchKernelGGL((moe_down_tiles_kernel<SPB, RT, WIDE, ZEROS>), dim3(oz2_w4_compute_units() * kMoeFit), dim3(64 * kMoeWaves), kMoeLds, c.st, c, scale_type);
}
template <int SPB, int RT>
void launch_down_tiles(const MoeCall& c, int scale_type) {
  if (scale_type == OZ2_F32) c.down.zeros ? launch_down_tiles<SPB, RT, true, true>(c, scale_type) : launch_down_tiles<SPB, RT, true, false>(c, scale_type);
  else c.down.zeros ? launch_down_tiles<SPB, RT, false, true>(c, scale_type) : launch_down_tiles<SPB, RT, false, false>(c, scale_type);
}
template <int SPB>
void launch_down_tiles(const MoeCall& c, int scale_type) {
  if (c.tiles == 4) launch_down_tiles<SPB, 1>(c, scale_type);
  else launch_down_tiles<SPB, 4>(c, scale_type);
}

}  // namespace

hipError_t oz2_moe_down(const MoeCall& c, const oz2_w4_matrix& down) {
  const int type = down.scale_type;
  if (c.tiles == 1) {
    if (type == OZ2_F32) launch_down<OZ2_F32>(c);
    else if (type == OZ2_BF16) launch_down<OZ2_BF16>(c);
    else launch_down<OZ2_F16>(c);
  } else {
    if (down.group == 32) launch_down_tiles<4>(c, type);
    else if (down.group == 64) launch_down_tiles<2>(c, type);
    else launch_down_tiles<1>(c, type);
  }
  if (c.tiles > 1 || !c.direct) hipLaunchKernelGGL(moe_sum_kernel, dim3((c.d + 255) / 256, c.t), dim3(256), 0, c.st, c);
  return hipGetLastError();
}
