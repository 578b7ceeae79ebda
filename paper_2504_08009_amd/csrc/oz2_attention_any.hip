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

template <int XT, int DP>
__global__ void __launch_bounds__(256) attention_any_kernel(Attention a) {
  constexpr int E = DP / 8, F = DP / 32;
  __shared__ float merged[4 * kRows * (DP + 1)];  // [wave][row][DP + 1]
  __shared__ float merged_m[4][kRows], merged_l[4][kRows];
  const AttentionTile tile = attention_tile(a, blockIdx.x, kRows);
  const int rows = tile.tokens * a.group;
  if (tile.first >= rows) return;
  const int head = blockIdx.y, lane = threadIdx.x % 64, wave = threadIdx.x / 64, col = lane % 32, half = lane / 32;
  const int row = min(tile.first + col, rows - 1), at = row / a.per_group;
  const int64_t query = (int64_t)head * a.group + (row - at * a.group);
  const int sees = a.causal ? at + 1 : tile.tokens;

  float q[E][4];  // dims 8 e + 4 half + j
  for (int e = 0; e < E; ++e)
    for (int j = 0; j < 4; ++j) {
      const int d = 8 * e + 4 * half + j;
      q[e][j] = d < a.dim ? w4_load(XT, a.q.data, (tile.begin + at) * a.q.ld_token + query * a.q.ld_head + d) : 0.f;
    }
  float m = -3e38f, l = 0.f;
  f16v o[F];
  for (int f = 0; f < F; ++f)
    for (int i = 0; i < 16; ++i) o[f][i] = 0.f;

  // keys that any row of the tile sees
  const int end = a.causal ? min(tile.first + kRows - 1, rows - 1) / a.per_group + 1 : tile.tokens;
  for (int k0 = wave * kKeys; k0 < end; k0 += 4 * kKeys) {
    f16v s;
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
    const int64_t key = tile.begin + min(k0 + col, tile.tokens - 1);
    for (int e = 0; e < E; ++e) {
      if (8 * e >= a.dim) break;
      for (int j = 0; j < 4; ++j) {
        const int d = 8 * e + 4 * half + j;
        const float k = d < a.dim ? w4_load(XT, a.k.data, key * a.k.ld_token + head * a.k.ld_head + d) : 0.f;
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(k, q[e][j], s, 0, 0, 0);
      }
    }
    float high = -INFINITY;
    for (int i = 0; i < 16; ++i) {
      const int place = k0 + i / 4 * 8 + i % 4 + 4 * half;
      if (place >= sees) s[i] = -INFINITY;
      s[i] *= a.scale2;
      high = fmaxf(high, s[i]);
    }
    high = fmaxf(high, __shfl_xor(high, 32));
    const float raised = fmaxf(m, high), factor = __builtin_amdgcn_exp2f(m - raised);
    m = raised;
    l *= factor;
    for (int f = 0; f < F; ++f) o[f] *= factor;
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(s[i] - m);
      l += s[i];
    }
    // values that a row does not see must not reach it, not even as 0 times an infinity: where a tile has both, such values are taken apart
    const bool partly = a.causal && k0 + kKeys > tile.first / a.per_group + 1;
    for (int i = 0; i < 16; ++i) {
      const int place = k0 + i / 4 * 8 + i % 4 + 4 * half;
      const bool there = place < end;  // (those behind are seen by no row)
      const int64_t value = tile.begin + min(place, tile.tokens - 1);
      for (int f = 0; f < F; ++f) {
        const int d = 32 * f + col;
        float v = there && d < a.dim ? w4_load(XT, a.v.data, value * a.v.ld_token + head * a.v.ld_head + d) : 0.f;
        if (partly) {
          const bool odd = !(fabsf(v) < INFINITY);
          if (__any(odd)) {
            for (unsigned long long left = __ballot(odd); left; left &= left - 1) {
              const int from = __ffsll((long long)left) - 1;  // the lane that has dim 32 f + from % 32 of its place
              const float bad = __shfl(v, from), p = __shfl(s[i], from / 32 * 32 + col);
              const int bad_place = k0 + i / 4 * 8 + i % 4 + 4 * (from / 32), in = from % 32;
              // the lane and register of the row's sum: dim in = 8 (r / 4) + 4 half + r % 4
              if (bad_place < sees && half == in / 4 % 2)
                for (int r = 0; r < 16; ++r)
                  if (r == in / 8 * 4 + in % 4) o[f][r] = fmaf(p, bad, o[f][r]);
            }
            if (odd) v = 0.f;
          }
        }
        o[f] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[i], o[f], 0, 0, 0);
      }
    }
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
  hipLaunchKernelGGL((attention_any_kernel<XT, DP>), dim3((unsigned)attention_tiles(a, kRows), (unsigned)a.kv_heads), dim3(256), 0, st, a);
  return hipGetLastError();
}
template <int XT>
hipError_t of(const Attention& a, hipStream_t st) {
  return a.dim <= 64 ? launch<XT, 64>(a, st) : a.dim <= 128 ? launch<XT, 128>(a, st) : launch<XT, 256>(a, st);
}

}  // namespace

hipError_t oz2_attention_any(const Attention& a, hipStream_t st) {
  return a.q.type == OZ2_F32 ? of<OZ2_F32>(a, st) : a.q.type == OZ2_BF16 ? of<OZ2_BF16>(a, st) : of<OZ2_F16>(a, st);
}
