// Attention over packed prompts for any type, dim up to 256 and strides, in FP32 throughout.
//
// A workgroup has 32 rows; its four waves take tiles of 32 keys in turn, each with sums and a maximum of its own, which come together at the end.  Products are
// keys x rows and dims x rows on the FP32 matrix cores (32 x 32 x 2), so that a lane has one row throughout, and what it holds of the first product is what the
// second one wants of it: places 8 (i / 4) + i % 4 and, in the upper half of the lanes, four further on.  Keys and values are read by the lanes that need
// them, from the caches.
#include "oz2_attention.h"

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));
constexpr int kRows = 32, kKeys = 32;

// N values beside each other, in FP32
template <int XT, int N>
__device__ __forceinline__ void values(const char* p, float (&x)[N]) {
  if constexpr (N == 1) x[0] = w4_load(XT, p, 0);
  else if constexpr (XT == OZ2_F32) {
    struct __attribute__((packed, aligned(4))) Four { float v[4]; };
    const Four f = *reinterpret_cast<const Four*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = f.v[j];
  } else {
    struct __attribute__((packed, aligned(2))) Four { uint16_t v[4]; };
    const Four f = *reinterpret_cast<const Four*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (XT == OZ2_BF16) x[j] = __uint_as_float((unsigned)f.v[j] << 16);
      else x[j] = (float)__builtin_bit_cast(_Float16, f.v[j]);
    }
  }
}

// FOURS: dim is a multiple of four
template <int XT, int DP, bool FOURS>
__global__ void __launch_bounds__(256, 1) attention_any_kernel(Attention a) {
  constexpr int E = DP / 8, F = DP / 32, SIZE = XT == OZ2_F32 ? 4 : 2;
  __shared__ float merged[4 * kRows * (DP + 1)];  // [wave][row][DP + 1]
  __shared__ float merged_m[4][kRows], merged_l[4][kRows];
  const AttentionTile tile = attention_tile(a, blockIdx.x, gridDim.x, kRows);
  const int rows = tile.tokens * a.group;
  if (tile.first >= rows) return;
  const int head = blockIdx.y, lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 32, half = lane / 32;
  const int row = min(tile.first + col, rows - 1), at = row / a.per_group;
  const int64_t query = (int64_t)head * a.group + (row - at * a.group);
  const int sees = a.causal ? at + 1 : tile.tokens;

  float q[E][4];  // dims 8 e + 4 half + j
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = 8 * e + 4 * half + j;
      q[e][j] = d < a.dim ? w4_load(XT, a.q.data, (tile.begin + at) * a.q.ld_token + query * a.q.ld_head + d) : 0.f;
    }
  float m = -3e38f, l = 0.f;
  f16v o[F];
#pragma unroll
  for (int f = 0; f < F; ++f)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[f][i] = 0.f;

  const char* k_from = static_cast<const char*>(a.k.data) + (tile.begin * a.k.ld_token + head * a.k.ld_head) * SIZE;
  const char* v_from = static_cast<const char*>(a.v.data) + (tile.begin * a.v.ld_token + head * a.v.ld_head) * SIZE;
  // (a dim that is not there: of keys another one, which meets a 0 of q; of values another one, whose sum is not stored)
  auto keys = [&](int k0, float (&k)[E][4]) {
    const char* from = k_from + min(k0 + col, tile.tokens - 1) * a.k.ld_token * SIZE;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int d = 8 * e + 4 * half;
      if constexpr (FOURS) values<XT, 4>(from + (d < a.dim ? d : 0) * SIZE, k[e]);
      else {
#pragma unroll
        for (int j = 0; j < 4; ++j) k[e][j] = w4_load(XT, from, d + j < a.dim ? d + j : 0);
      }
    }
  };

  // keys that any row of the tile sees
  const int end = a.causal ? min(tile.first + kRows - 1, rows - 1) / a.per_group + 1 : tile.tokens;
  float k[E][4], v[16][F];
  if (wave * kKeys < end) keys(wave * kKeys, k);
  for (int k0 = wave * kKeys; k0 < end; k0 += 4 * kKeys) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const char* from = v_from + min(k0 + i / 4 * 8 + i % 4 + 4 * half, tile.tokens - 1) * a.v.ld_token * SIZE;
#pragma unroll
      for (int f = 0; f < F; ++f) v[i][f] = w4_load(XT, from, 32 * f + col < a.dim ? 32 * f + col : 0);
    }
    f16v s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e][j], q[e][j], s, 0, 0, 0);
    if (k0 + 4 * kKeys < end) keys(k0 + 4 * kKeys, k);
    float high = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int place = k0 + i / 4 * 8 + i % 4 + 4 * half;
      s[i] = place >= sees ? -INFINITY : s[i] * a.scale2;
      high = fmaxf(high, s[i]);
    }
    high = fmaxf(high, __shfl_xor(high, 32));
    const float raised = fmaxf(m, high), factor = __builtin_amdgcn_exp2f(m - raised);
    m = raised;
    l *= factor;
#pragma unroll
    for (int f = 0; f < F; ++f) o[f] *= factor;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(s[i] - m);
      l += s[i];
    }
    if (k0 + kKeys > end) {  // places that no row sees
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int f = 0; f < F; ++f) v[i][f] = k0 + i / 4 * 8 + i % 4 + 4 * half < end ? v[i][f] : 0.f;
    }
    // Values that a row does not see must not reach it, not even as 0 times an infinity: where a tile has both, such values are taken apart.
    if (a.causal && k0 + kKeys > tile.first / a.per_group + 1) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int f = 0; f < F; ++f) {
          const bool odd = !(fabsf(v[i][f]) < INFINITY);
          for (unsigned long long left = __ballot(odd); left; left &= left - 1) {
            const int from = __ffsll((long long)left) - 1;  // the lane that has dim 32 f + from % 32 of its place
            const float bad = __shfl(v[i][f], from), p = __shfl(s[i], from / 32 * 32 + col);
            const int bad_place = k0 + i / 4 * 8 + i % 4 + 4 * (from / 32), in = from % 32;
            // the lane and register of the row's sum: dim in = 8 (r / 4) + 4 half + r % 4
            if (bad_place < sees && half == in / 4 % 2)
              for (int r = 0; r < 16; ++r)
                if (r == in / 8 * 4 + in % 4) o[f][r] = fmaf(p, bad, o[f][r]);
          }
          v[i][f] = odd ? 0.f : v[i][f];
        }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int f = 0; f < F; ++f) o[f] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[i][f], s[i], o[f], 0, 0, 0);
  }
  l += __shfl_xor(l, 32);
  if (half == 0) merged_m[wave][col] = m, merged_l[wave][col] = l;
  for (int f = 0; f < F; ++f)
    for (int i = 0; i < 16; ++i) merged[(wave * kRows + col) * (DP + 1) + 32 * f + i / 4 * 8 + i % 4 + 4 * half] = o[f][i];
  __syncthreads();
  for (int i = threadIdx.x; i < kRows * DP; i += 256) {
    const int r = i / DP, d = i % DP;
    if (tile.first + r >= rows || d >= a.dim) continue;
    float high = merged_m[0][r], total = 0.f, v = 0.f;
    for (int w = 1; w < 4; ++w) high = fmaxf(high, merged_m[w][r]);
    for (int w = 0; w < 4; ++w) {
      const float factor = __builtin_amdgcn_exp2f(merged_m[w][r] - high);
      total = fmaf(factor, merged_l[w][r], total);
      v = fmaf(factor, merged[(w * kRows + r) * (DP + 1) + d], v);
    }
    const int of = (tile.first + r) / a.per_group;
    w4_store(a.out.type, a.out.data, (tile.begin + of) * a.out.ld_token + ((int64_t)head * a.group + (tile.first + r - of * a.group)) * a.out.ld_head + d,
             total == 0.f ? 0.f : v / total);
  }
}

template <int XT, int DP>
hipError_t launch(const Attention& a, hipStream_t st) {
  const dim3 grid((unsigned)attention_tiles(a, kRows), (unsigned)a.kv_heads);
  if (a.dim % 4 == 0) hipLaunchKernelGGL((attention_any_kernel<XT, DP, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((attention_any_kernel<XT, DP, false>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}
template <int XT>
hipError_t of(const Attention& a, hipStream_t st) {
  return a.dim <= 64 ? launch<XT, 64>(a, st) : a.dim <= 96 ? launch<XT, 96>(a, st) : a.dim <= 128 ? launch<XT, 128>(a, st) : launch<XT, 256>(a, st);
}

}  // namespace

hipError_t oz2_attention_any(const Attention& a, hipStream_t st) {
  return a.q.type == OZ2_F32 ? of<OZ2_F32>(a, st) : a.q.type == OZ2_BF16 ? of<OZ2_BF16>(a, st) : of<OZ2_F16>(a, st);
}
