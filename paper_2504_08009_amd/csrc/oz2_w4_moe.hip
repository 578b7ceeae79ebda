// A layer of gated experts whose weights are held in 4 bits, with its router, for a few tokens (oz2_w4_moe).
#include "oz2_w4.h"

namespace {

__device__ __forceinline__ float wave_sum(float v) {
  for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
  return v;
}

// One wave a logit.
__global__ void __launch_bounds__(256) moe_logits_kernel(oz2_moe_layer m, int x_type, const char* x, int64_t ldx, float* logits) {
  const int64_t e = (int64_t)blockIdx.x * 4 + threadIdx.x / 64, t = blockIdx.y;
  const int lane = threadIdx.x % 64;
  if (e >= m.gate.count) return;
  float sum = 0.f;
  for (int64_t i = lane; i < m.gate.k; i += 64)
    sum = fmaf(w4_load(m.router_type, m.router, e * m.ld_router + i), w4_load(x_type, x, t * ldx + i), sum);
  sum = wave_sum(sum);
  if (lane == 0) logits[t * m.gate.count + e] = sum;
}

// One thread a token.
__global__ void moe_choose_kernel(oz2_moe_layer m, int64_t t, const uint8_t* active, const float* logits, int* ids, float* weights) {
  const int64_t i = (int64_t)blockIdx.x * 64 + threadIdx.x;
  if (i >= t) return;
  const int count = (int)m.gate.count;
  const float* l = logits + i * count;
  float high = -INFINITY, total = 0.f;
  for (int e = 0; e < count; ++e) high = fmaxf(high, l[e]);
  for (int e = 0; e < count; ++e) total += expf(l[e] - high);
  auto score = [&](int e) { return m.score == OZ2_SCORE_SOFTMAX ? expf(l[e] - high) / total : 1.f / (1.f + expf(-l[e])); };
  float last = INFINITY, sum = 0.f;
  int last_id = -1;
  for (int j = 0; j < m.top_k; ++j) {
    float best = -INFINITY;
    int id = -1;
    for (int e = 0; e < count; ++e) {
      float key = score(e) + (m.bias ? m.bias[e] : 0.f);
      if (key != key) key = INFINITY;
      if ((key < last || (key == last && e > last_id)) && key > best) best = key, id = e;
    }
    if (active && !active[i]) id = -1;
    ids[i * m.top_k + j] = id;
    const float p = id >= 0 ? score(id) : 0.f;
    weights[i * m.top_k + j] = p;
    sum += p;
    last = best, last_id = id;
    if (id < 0) last = -INFINITY, last_id = count;
  }
  for (int j = 0; j < m.top_k; ++j) {
    float p = weights[i * m.top_k + j];
    if (m.renormalize) p = sum == 0.f ? 0.f : p / sum;
    weights[i * m.top_k + j] = p * m.factor;
  }
}

__device__ float w4_row_times(const oz2_w4_matrix& w, int64_t e, int64_t row, int type, const void* x, int64_t at, int lane) {
  const uint8_t* codes = static_cast<const uint8_t*>(w.codes) + e * w.stride_codes + row * w.ld_codes;
  float sum = 0.f;
  for (int64_t l = lane; l < w.k; l += 64) {
    const int q = codes[l / 2] >> (l % 2 * 4) & 15;
    const int64_t g = l / w.group;
    const int z = w.zeros ? static_cast<const uint8_t*>(w.zeros)[e * w.stride_zeros + row * w.ld_zeros + g] : 8;
    sum = fmaf(w4_load(w.scale_type, w.scales, e * w.stride_scales + row * w.ld_scales + g) * (float)(q - z), w4_load(type, x, at + l), sum);
  }
  return wave_sum(sum);
}

// One wave an inner value of a place (a token's j-th expert).
__global__ void __launch_bounds__(256) moe_inner_kernel(oz2_moe_layer m, int x_type, const char* x, int64_t ldx, const int* ids, float* h) {
  const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64, place = blockIdx.y;
  const int lane = threadIdx.x % 64, e = ids[place];
  if (row >= m.gate.n || e < 0) return;
  const int64_t at = place / m.top_k * ldx;
  const float g = w4_row_times(m.gate, e, row, x_type, x, at, lane), u = w4_row_times(m.up, e, row, x_type, x, at, lane);
  const float a = m.activation == OZ2_ACT_SILU ? g / (1.f + expf(-g)) : 0.5f * g * (1.f + erff(g * 0.70710678f));
  if (lane == 0) h[place * m.gate.n + row] = a * u;
}

// One wave an output.
__global__ void __launch_bounds__(256) moe_outer_kernel(oz2_moe_layer m, const int* ids, const float* weights, const float* h, int y_type, char* y,
                                                        int64_t ldy) {
  const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64, t = blockIdx.y;
  const int lane = threadIdx.x % 64;
  if (row >= m.down.n) return;
  float sum = 0.f;
  for (int j = 0; j < m.top_k; ++j) {
    const int64_t place = t * m.top_k + j;
    if (ids[place] >= 0) sum = fmaf(weights[place], w4_row_times(m.down, ids[place], row, OZ2_F32, h, place * m.gate.n, lane), sum);
  }
  if (lane == 0) w4_store(y_type, y, t * ldy + row, sum);
}

struct Space {
  size_t logits, ids, weights, h, total;
};
Space space(const oz2_moe_layer& m, int64_t t) {
  Space s;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) / 256 * 256; return o; };
  s.logits = take((size_t)t * m.gate.count * 4);
  s.ids = take((size_t)t * m.top_k * 4);
  s.weights = take((size_t)t * m.top_k * 4);
  s.h = take((size_t)t * m.top_k * m.gate.n * 4);
  s.total = at;
  return s;
}

}  // namespace

size_t oz2_w4_moe_space(const oz2_moe_layer& m, int64_t t) { return space(m, t).total; }

hipError_t oz2_launch_w4_moe(const oz2_moe_layer& m, int64_t t, int x_type, const void* x, int64_t ldx, const uint8_t* active, int y_type,
                             void* y, int64_t ldy, int32_t* ids, float* weights, char* ws, hipStream_t st) {
  const Space s = space(m, t);
  float* logits = reinterpret_cast<float*>(ws + s.logits);
  float* h = reinterpret_cast<float*>(ws + s.h);
  if (!ids) ids = reinterpret_cast<int32_t*>(ws + s.ids);
  if (!weights) weights = reinterpret_cast<float*>(ws + s.weights);
  const char* xp = static_cast<const char*>(x);
  hipLaunchKernelGGL(moe_logits_kernel, dim3((unsigned)((m.gate.count + 3) / 4), (unsigned)t), dim3(256), 0, st, m, x_type, xp, ldx, logits);
  hipLaunchKernelGGL(moe_choose_kernel, dim3((unsigned)((t + 63) / 64)), dim3(64), 0, st, m, t, active, logits, ids, weights);
  hipLaunchKernelGGL(moe_inner_kernel, dim3((unsigned)((m.gate.n + 3) / 4), (unsigned)(t * m.top_k)), dim3(256), 0, st, m, x_type, xp, ldx, ids, h);
  hipLaunchKernelGGL(moe_outer_kernel, dim3((unsigned)((m.down.n + 3) / 4), (unsigned)t), dim3(256), 0, st, m, ids, weights, h, y_type,
                     static_cast<char*>(y), ldy);
  return hipGetLastError();
}
