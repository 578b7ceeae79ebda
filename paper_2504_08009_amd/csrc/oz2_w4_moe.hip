// A layer of gated experts whose weights are held in 4 bits, with its router, for a few tokens (oz2_w4_moe).
#include "oz2_w4_moe.h"

#include <algorithm>

extern template hipError_t oz2_moe_gate_up<OZ2_F32>(const MoeCall&, const oz2_w4_matrix&);
extern template hipError_t oz2_moe_gate_up<OZ2_BF16>(const MoeCall&, const oz2_w4_matrix&);
extern template hipError_t oz2_moe_gate_up<OZ2_F16>(const MoeCall&, const oz2_w4_matrix&);

namespace {

__device__ __forceinline__ float wave_sum(float v) {
  for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
  return v;
}

// Logits of four tokens for an expert: a workgroup, whose waves share the inner dimension; a lane takes eight values of each at a time.
template <int TYPE>
__device__ __forceinline__ void load_eight(const char* p, int64_t i, int left, float (&out)[8]) {
  constexpr int size = TYPE == OZ2_F32 ? 4 : 2;
  if (left >= 8) {
    w4_u4 a = w4_bytes<16>(p + i * size), b = a;
    if constexpr (TYPE == OZ2_F32) b = w4_bytes<16>(p + (i + 4) * size);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (TYPE == OZ2_F32) out[e] = __uint_as_float(e < 4 ? a[e % 4] : b[e % 4]);
      else out[e] = w4_decode16(TYPE, a[e / 2] >> (e % 2 * 16) & 0xFFFFu);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = e < left ? w4_load(TYPE, p, i + e) : 0.f;
  }
}
template <int RT, int XT>
__global__ void __launch_bounds__(256) moe_router_kernel(const char* router, int64_t ld_router, MoeCall c) {
  __shared__ float part[4][4];
  const int e = blockIdx.x, wave = threadIdx.x / 64, lane = threadIdx.x % 64, first = blockIdx.y * 4, tokens = min(4, c.t - first);
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
  for (int i = threadIdx.x * 8; i < c.d; i += 2048) {
    float r[8], x[4][8];
    load_eight<RT>(router, e * ld_router + i, c.d - i, r);
#pragma unroll
    for (int t = 0; t < 4; ++t) load_eight<XT>(c.x, (first + min(t, tokens - 1)) * c.ldx + i, c.d - i, x[t]);
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[t] = fmaf(r[j], x[t][j], sum[t]);
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) sum[t] = wave_sum(sum[t]);
  if (lane == 0)
#pragma unroll
    for (int t = 0; t < 4; ++t) part[wave][t] = sum[t];
  __syncthreads();
  if (threadIdx.x < tokens)
    c.logits[(int64_t)(first + threadIdx.x) * c.experts + e] = (part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]);
}
template <int RT>
void launch_router(const oz2_moe_layer& m, int x_type, const MoeCall& c) {
  const dim3 grid(c.experts, (c.t + 3) / 4), block(256);
  const char* r = static_cast<const char*>(m.router);
  if (x_type == OZ2_F32) hipLaunchKernelGGL((moe_router_kernel<RT, OZ2_F32>), grid, block, 0, c.st, r, m.ld_router, c);
  else if (x_type == OZ2_BF16) hipLaunchKernelGGL((moe_router_kernel<RT, OZ2_BF16>), grid, block, 0, c.st, r, m.ld_router, c);
  else hipLaunchKernelGGL((moe_router_kernel<RT, OZ2_F16>), grid, block, 0, c.st, r, m.ld_router, c);
}

// The kernels below serve layers whose vectors are too short or too long for those of the other files.

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
  size_t logits, ids, weights, chosen, h, part, total;
};
Space space(const oz2_moe_layer& m, int64_t t) {
  Space s;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) / 256 * 256; return o; };
  const size_t at_once = t < kMoeTokens ? t : kMoeTokens, places = at_once * m.top_k;
  s.logits = take(at_once * m.gate.count * 4);
  s.ids = take(places * 4);
  s.weights = take(places * 4);
  s.chosen = take((2 + 3 * (size_t)kMoePlaces) * 4);
  s.h = take(places * m.gate.n * 4);
  s.part = take(places * m.down.n * 4);
  s.total = at;
  return s;
}

}  // namespace

int oz2_w4_compute_units() {
  static const int cus = [] {
    int device = 0, n = 0;
    return hipGetDevice(&device) == hipSuccess && hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, device) == hipSuccess && n > 0 ? n : 256;
  }();
  return cus;
}

size_t oz2_w4_moe_space(const oz2_moe_layer& m, int64_t t) { return space(m, t).total; }

hipError_t oz2_launch_w4_moe(const oz2_moe_layer& m, int64_t t, int x_type, const void* x, int64_t ldx, const uint8_t* active, int y_type,
                             void* y, int64_t ldy, int32_t* ids, float* weights, char* ws, hipStream_t st) {
  const Space s = space(m, t);
  const int64_t d = m.gate.k, f = m.gate.n;
  const int x_size = x_type == OZ2_F32 ? 4 : 2, y_size = y_type == OZ2_F32 ? 4 : 2;
  for (int64_t first = 0; first < t; first += kMoeTokens) {
    MoeCall c;
    c.t = (int)(t - first < kMoeTokens ? t - first : kMoeTokens);
    c.d = (int)d, c.f = (int)f, c.experts = (int)m.gate.count, c.top_k = m.top_k;
    c.score = m.score, c.renormalize = m.renormalize, c.activation = m.activation, c.factor = m.factor, c.bias = m.bias;
    c.active = active ? active + first : nullptr;
    c.x = static_cast<const char*>(x) + first * ldx * x_size, c.ldx = ldx;
    const oz2_w4_matrix* of[3] = {&m.gate, &m.up, &m.down};
    W4Rows* rows[3] = {&c.gate, &c.up, &c.down};
    for (int i = 0; i < 3; ++i) {
      *rows[i] = oz2_w4_rows(*of[i]);
      c.code_strides[i] = of[i]->stride_codes, c.scale_strides[i] = of[i]->stride_scales * (of[i]->scale_type == OZ2_F32 ? 4 : 2);
      c.zero_strides[i] = of[i]->stride_zeros;
    }
    c.y_type = y_type, c.y = static_cast<char*>(y) + first * ldy * y_size, c.ldy = ldy;
    c.logits = reinterpret_cast<float*>(ws + s.logits);
    c.ids = ids ? ids + first * m.top_k : reinterpret_cast<int32_t*>(ws + s.ids);
    c.weights = weights ? weights + first * m.top_k : reinterpret_cast<float*>(ws + s.weights);
    c.chosen = reinterpret_cast<int*>(ws + s.chosen);
    c.h = reinterpret_cast<float*>(ws + s.h), c.part = reinterpret_cast<float*>(ws + s.part);
    // Matrix cores or vector units.  Above two tokens for an expert on the average: the matrix cores, up to 16 (FP32: 12) at a time.  From a half to two, up
    // to 4 at a time, and only where every compute unit gets a workgroup of either product: a wave that has 32 rows to itself takes long.  Layers
    // of D x F, us by the vector units / the matrix cores:
    //   load 0.53 (8 tokens, 4 of 60 experts, 2048 x 1024, FP32) 54 / 49, 0.75 (12, 4 of 64, 2048 x 2048) 96 / 80, 1 (16, 8 of 128, 4096 x 2048)
    //   339 / 267, 1.5 (16, 6 of 64, 2048 x 1408) 142 / 88, 2 (32, 8 of 128, 4096 x 2048) 657 / 376, 2.9 (23, 2 of 16, 3000 x 1500) 144 / 83,
    //   4 (32, 8 of 64, 2048 x 1024) 222 / 90, 16 (32, 4 of 8, 4096 x 2048) 307 / 126;
    //   few workgroups: 1 (2, 2 of 4, 4096 x 2048) 32 / 48, 1 (8, 1 of 8, 1000 x 4096) 34 / 53, 2 (8, 2 of 8, 2048 x 4096) 60 / 76.
    const bool near = w4_tile_fits(c.gate) && w4_tile_fits(c.up) && w4_tile_fits(c.down);
    const int places = c.t * c.top_k, of_expert = std::min((c.f + 63) / 64, (c.d + 127) / 128);
    const bool filled = std::min(places, c.experts) * of_expert >= oz2_w4_compute_units();
    c.tiles = !near || 2 * places <= c.experts ? 1 : places > 2 * c.experts ? 16 : filled ? 4 : 1;
    // Hardly an expert with two tokens: each token's second products are summed where they are formed.
    c.direct = c.t == 1 || 2 * places <= c.experts;
    c.st = st;
    // rows of 16 bytes of codes or more, and spans of 2048 for the waves of a workgroup
    if (d < kW4Unit || f < kW4Unit || d > kMoeLongest || f > kMoeLongest) {
      hipLaunchKernelGGL(moe_logits_kernel, dim3((unsigned)((c.experts + 3) / 4), c.t), dim3(256), 0, st, m, x_type, c.x, ldx, c.logits);
      hipLaunchKernelGGL(moe_choose_kernel, dim3(1), dim3(64), 0, st, m, c.t, c.active, c.logits, c.ids, c.weights);
      hipLaunchKernelGGL(moe_inner_kernel, dim3((unsigned)((f + 3) / 4), c.t * c.top_k), dim3(256), 0, st, m, x_type, c.x, ldx, c.ids, c.h);
      hipLaunchKernelGGL(moe_outer_kernel, dim3((unsigned)((d + 3) / 4), c.t), dim3(256), 0, st, m, c.ids, c.weights, c.h, y_type, c.y, ldy);
      if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
      continue;
    }
    if (m.router_type == OZ2_F32) launch_router<OZ2_F32>(m, x_type, c);
    else if (m.router_type == OZ2_BF16) launch_router<OZ2_BF16>(m, x_type, c);
    else launch_router<OZ2_F16>(m, x_type, c);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess)
      e = x_type == OZ2_F32    ? oz2_moe_gate_up<OZ2_F32>(c, m.gate)
          : x_type == OZ2_BF16 ? oz2_moe_gate_up<OZ2_BF16>(c, m.gate)
                               : oz2_moe_gate_up<OZ2_F16>(c, m.gate);
    if (e == hipSuccess) e = oz2_moe_down(c, m.down);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
