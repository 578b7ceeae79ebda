// Choice of the experts and their first products: h = act(gate x) * (up x) for every place.
#ifndef OZ2_W4_MOE_UP_H
#define OZ2_W4_MOE_UP_H

#include "oz2_w4_moe.h"

#ifdef __HIPCC__
namespace {

// Over the wave, in every lane.
__device__ __forceinline__ float wave_max(float v) {
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  auto larger = [](u2 r) { return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])); };
  v = fmaxf(v, w4_partner<0>(v)), v = fmaxf(v, w4_partner<1>(v)), v = fmaxf(v, w4_partner<2>(v)), v = fmaxf(v, w4_partner<3>(v));
  v = larger(__builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false));
  return larger(__builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
}
__device__ __forceinline__ float wave_sum(float v) {
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  auto both = [](u2 r) { return __uint_as_float(r[0]) + __uint_as_float(r[1]); };
  v += w4_partner<0>(v), v += w4_partner<1>(v), v += w4_partner<2>(v), v += w4_partner<3>(v);
  v = both(__builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false));
  return both(__builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
}

// Experts and weights of one token, by one wave; ids (LDS) gets -1 where there is none.  A lane holds V neighbouring experts, so that the
// first lane with the largest key has the lowest index that has it.
template <int V>
__device__ __forceinline__ void moe_choose(const MoeCall& c, int token, short* ids, float* weights) {
  const int lane = threadIdx.x % 64;
  const float* logits = c.logits + (int64_t)token * c.experts;
  float p[V], key[V], high = -INFINITY;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = lane * V + i;
    p[i] = e < c.experts ? logits[e] : -INFINITY;
    key[i] = e < c.experts && c.bias ? c.bias[e] : 0.f;
    high = fmaxf(high, p[i]);
  }
  if (c.score == OZ2_SCORE_SOFTMAX) {
    float total = 0.f;
    high = wave_max(high);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      p[i] = lane * V + i < c.experts ? expf(p[i] - high) : 0.f;
      total += p[i];
    }
    total = wave_sum(total);
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] /= total;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = 1.f / (1.f + expf(-p[i]));
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    key[i] = lane * V + i < c.experts ? p[i] + key[i] : -INFINITY;
    if (key[i] != key[i]) key[i] = INFINITY;
  }
  const bool active = !c.active || c.active[token];
  float sum = 0.f, mine = 0.f;  // (lane j keeps the j-th)
  int id = -1;
  for (int j = 0; j < c.top_k; ++j) {
    float best = key[0];
#pragma unroll
    for (int i = 1; i < V; ++i) best = fmaxf(best, key[i]);
    const float most = wave_max(best);
    if (!active || !(most > -INFINITY)) break;
    const int winner = __ffsll(__ballot(best == most)) - 1;
    float w = 0.f;
    int which = -1;
#pragma unroll
    for (int i = V - 1; i >= 0; --i)
      if (key[i] == most) w = p[i], which = i;
    w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), winner));
    which = __builtin_amdgcn_readlane(which, winner);
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (lane == winner && i == which) key[i] = -INFINITY;
    sum += w;
    if (lane == j) mine = w, id = winner * V + which;
  }
  if (c.renormalize) mine = sum == 0.f ? 0.f : mine / sum;
  if (lane < c.top_k) {
    ids[token * c.top_k + lane] = id;
    weights[token * c.top_k + lane] = mine * c.factor;
  }
}

// Every workgroup makes the choice for itself, which is cheaper than a launch in between; the first one leaves it for the launches behind.
__device__ __forceinline__ void moe_route(const MoeCall& c, Chosen& chosen, short* ids, float* weights, int* count) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int places = c.t * c.top_k;
  auto choose = [&](int token) {
    if (c.experts <= 64) moe_choose<1>(c, token, ids, weights);
    else if (c.experts <= 128) moe_choose<2>(c, token, ids, weights);
    else if (c.experts <= 256) moe_choose<4>(c, token, ids, weights);
    else moe_choose<16>(c, token, ids, weights);
  };
  if (c.t == 1) {  // every place has an expert of its own, and those without one come last
    if (wave == 0) {
      choose(0);
      const int id = lane < c.top_k ? ids[lane] : -1, n = __popcll(__ballot(id >= 0));
      if (id >= 0) chosen.expert[lane] = id, chosen.place[lane] = lane;
      if (lane <= n) chosen.first[lane] = lane;
      if (lane == 0) chosen.count = n;
      if (blockIdx.x == 0) {
        if (lane < c.top_k) c.ids[lane] = id, c.weights[lane] = weights[lane];
        if (lane == 0) c.chosen[0] = n;
        if (lane <= n) c.chosen[1 + lane] = lane;
        if (id >= 0) c.chosen[2 + kMoePlaces + lane] = id, c.chosen[2 + 2 * kMoePlaces + lane] = lane;
      }
    }
    __syncthreads();
    return;
  }
  for (int e = threadIdx.x; e < c.experts; e += 64 * kMoeWaves) count[e] = 0;
  for (int token = wave; token < c.t; token += kMoeWaves) choose(token);
  __syncthreads();
  for (int i = threadIdx.x; i < places; i += 64 * kMoeWaves)
    if (ids[i] >= 0) atomicAdd(&count[ids[i]], 1);
  __syncthreads();
  if (wave == 0) {  // experts that have places, and where these begin
    int found = 0, at = 0;
    for (int e = 0; e < c.experts; e += 64) {
      const int n = e + lane < c.experts ? count[e + lane] : 0;
      int before = n;
      for (int d = 1; d < 64; d *= 2) {
        const int other = __shfl_up(before, d);
        if (lane >= d) before += other;
      }
      const unsigned long long mask = __ballot(n > 0);
      if (n) {
        const int i = found + __popcll(mask & ((1ull << lane) - 1));
        chosen.expert[i] = e + lane;
        chosen.first[i] = at + before - n;
        count[e + lane] = at + before - n;  // from here on: where its next place goes
      }
      found += __popcll(mask);
      at += __shfl(before, 63);
    }
    if (lane == 0) chosen.count = found, chosen.first[found] = at;
  }
  __syncthreads();
  // (the order of an expert's places, which timing decides, changes no result: each is summed by itself, in an order that those beside it do not touch)
  for (int i = threadIdx.x; i < places; i += 64 * kMoeWaves)
    if (ids[i] >= 0) chosen.place[atomicAdd(&count[ids[i]], 1)] = i;
  __syncthreads();
  if (blockIdx.x) return;
  for (int i = threadIdx.x; i < places; i += 64 * kMoeWaves) c.ids[i] = ids[i], c.weights[i] = weights[i];
  int* to = c.chosen;
  const int n = chosen.count;
  if (threadIdx.x == 0) to[0] = n;
  for (int i = threadIdx.x; i <= n; i += 64 * kMoeWaves) to[1 + i] = chosen.first[i];
  for (int i = threadIdx.x; i < n; i += 64 * kMoeWaves) to[2 + kMoePlaces + i] = chosen.expert[i];
  for (int i = threadIdx.x; i < chosen.first[n]; i += 64 * kMoeWaves) to[2 + 2 * kMoePlaces + i] = chosen.place[i];
}

struct GateUp {
  W4Rows gate, up;
};
__device__ __forceinline__ GateUp moe_gate_up_of(const MoeCall& c, int64_t e) {
  return {w4_of_stack(c.gate, e, c.code_strides[0], c.scale_strides[0], c.zero_strides[0]),
          w4_of_stack(c.up, e, c.code_strides[1], c.scale_strides[1], c.zero_strides[1])};
}
__device__ __forceinline__ void moe_inner(const MoeCall& c, int place, int row, float g, float u) {
  if (row >= c.f) return;
  const float a = c.activation == OZ2_ACT_SILU ? g / (1.f + expf(-g)) : 0.5f * g * (1.f + erff(g * 0.70710678f));
  c.h[(int64_t)place * c.f + row] = a * u;
}

// One place of an expert at a time, by the vector units.
template <int XT, int ST, bool ZEROS, int FOLD>
__global__ void __launch_bounds__(64 * kMoeWaves, 4) moe_up_kernel(MoeCall c, int split_log) {
  __shared__ Chosen chosen;
  __shared__ short ids[kMoePlaces];
  __shared__ float weights[kMoePlaces];
  __shared__ int count[OZ2_MOE_MAX_EXPERTS];
  __shared__ float part[2][kMoeRounds][kMoeWaves][4 * FOLD];
  moe_route(c, chosen, ids, weights, count);
  moe_products<XT, ST, ZEROS, FOLD>(
      chosen, c.d, c.f, 2, split_log, c.gate, part, [&](int64_t e) { return moe_gate_up_of(c, e); },
      [&](const GateUp& m, int row, int i) { return w4_row<ST, FOLD>(i < 2 ? m.gate : m.up, row, i % 2); },
      [&](int place) { return c.x + place / c.top_k * c.ldx * (XT == OZ2_F32 ? 4 : 2); },
      [&](int place, int row, const float* u) {
#pragma unroll
        for (int i = 0; i < 2 * FOLD; ++i) moe_inner(c, place, row + i, u[i], u[2 * FOLD + i]);
      });
}

// Several, by the matrix cores: a tile of either matrix.
template <int XT, int SPB, int RT, bool WIDE, bool ZEROS>
__global__ void __launch_bounds__(64 * kMoeWaves, kMoeFit) moe_up_tiles_kernel(MoeCall c, int scale_type) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ Chosen chosen;
  {  // (the choice is done with its own arrays before x is brought in)
    short* ids = reinterpret_cast<short*>(lds);
    float* weights = reinterpret_cast<float*>(ids + kMoePlaces);
    moe_route(c, chosen, ids, weights, reinterpret_cast<int*>(weights + kMoePlaces));
    __syncthreads();
  }
  moe_tiles<XT, SPB, RT, WIDE, ZEROS>(
      chosen, c.t, c.d, c.f, 16, scale_type, lds, [&](int64_t e) { return moe_gate_up_of(c, e); },
      [](const GateUp& m, int t) { return t ? m.up : m.gate; }, [](int row, int) { return row; },
      [&](int place) { return c.x + place / c.top_k * c.ldx * (XT == OZ2_F32 ? 4 : 2); },
      [&](int place, int row, float g, float u) { moe_inner(c, place, row, g, u); });
}

template <int XT, int ST>
hipError_t launch_up(const MoeCall& c) {
  const dim3 grid(oz2_w4_compute_units() * 4), block(64 * kMoeWaves);
  const bool fold = moe_fold(c.gate) && moe_fold(c.up);
  const int split = fold ? 0 : moe_split(c.d);
  if (c.gate.zeros) {
    if (fold) hipLaunchKernelGGL((moe_up_kernel<XT, ST, true, 2>), grid, block, 0, c.st, c, split);
    else hipLaunchKernelGGL((moe_up_kernel<XT, ST, true, 1>), grid, block, 0, c.st, c, split);
  } else {
    if (fold) hipLaunchKernelGGL((moe_up_kernel<XT, ST, false, 2>), grid, block, 0, c.st, c, split);
    else hipLaunchKernelGGL((moe_up_kernel<XT, ST, false, 1>), grid, block, 0, c.st, c, split);
  }
  return hipGetLastError();
}

template <int XT, int SPB, int RT, bool WIDE, bool ZEROS>
hipError_t launch_up_tiles(const MoeCall& c, int scale_type) {
  hipLaunchKernelGGL((moe_up_tiles_kernel<XT, SPB, RT, WIDE, ZEROS>), dim3(oz2_w4_compute_units() * kMoeFit), dim3(64 * kMoeWaves), kMoeLds, c.st, c, scale_type);
  return hipGetLastError();
}
template <int XT, int SPB, int RT>
hipError_t launch_up_tiles(const MoeCall& c, int scale_type) {
  if (scale_type == OZ2_F32) return c.gate.zeros ? launch_up_tiles<XT, SPB, RT, true, true>(c, scale_type) : launch_up_tiles<XT, SPB, RT, true, false>(c, scale_type);
  return c.gate.zeros ? launch_up_tiles<XT, SPB, RT, false, true>(c, scale_type) : launch_up_tiles<XT, SPB, RT, false, false>(c, scale_type);
}
template <int XT, int SPB>
hipError_t launch_up_tiles(const MoeCall& c, int scale_type) {
  return c.tiles == 4 ? launch_up_tiles<XT, SPB, 1>(c, scale_type) : launch_up_tiles<XT, SPB, 4>(c, scale_type);
}

}  // namespace

template <int XT>
hipError_t oz2_moe_gate_up(const MoeCall& c, const oz2_w4_matrix& gate) {
  const int type = gate.scale_type;
  if (c.tiles == 1) return type == OZ2_F32 ? launch_up<XT, OZ2_F32>(c) : type == OZ2_BF16 ? launch_up<XT, OZ2_BF16>(c) : launch_up<XT, OZ2_F16>(c);
  return gate.group == 32 ? launch_up_tiles<XT, 4>(c, type) : gate.group == 64 ? launch_up_tiles<XT, 2>(c, type) : launch_up_tiles<XT, 1>(c, type);
}
#endif
#endif
