// New tokens' keys and values into a cache held in 4 bits (oz2_kv4_append): a vector of dim values becomes dim codes with a scale and an offset.
//
// A vector belongs to the smallest power of two of lanes that have eight values each, which is one word of codes a lane; smallest and largest value are found
// across lanes.  Bound by the bytes of k and v: 27100 tokens of 8 heads of 128 values, FP16, with what is held of them written too, take 58 us, 4.3 TB/s.
#include "oz2_kv4.h"
#include "oz2_fast_div.h"
#include "oz2_w4_core.h"

namespace {

struct Append {
  oz2_kv4_cache c;
  oz2_kv4_sequences on;
  const int32_t* at;
  oz2_rows x[2], held[2];
  int capacity, heads, page_size, lanes, total;
  FastDiv per_heads, per_page;
};

// over `lanes` neighbours, a power of two
template <class Op>
__device__ __forceinline__ float over(float v, int lanes, Op op) {
  auto with = [&](auto control) {
    return op(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), decltype(control)::value, 0xf, 0xf, true)));
  };
  if (lanes > 1) v = with(W4Index<0xb1>{});   // the neighbour
  if (lanes > 2) v = with(W4Index<0x4e>{});   // the other pair
  if (lanes > 4) v = with(W4Index<0x141>{});  // the other four, mirrored: all four have the same
  if (lanes > 8) v = with(W4Index<0x140>{});
  if (lanes > 16) v = op(v, __shfl_xor(v, 16));
  return v;
}

// N vectors a lane: their loads are under way together.  With one, a workgroup has all heads of some tokens; with more, runs of tokens of one head, which it
// writes beside each other.
template <int XT, int N>
__global__ void __launch_bounds__(256) kv4_append_kernel(Append a) {
  const int which = blockIdx.y;  // 0: keys, 1: values
  const int lane = threadIdx.x % a.lanes, step = 256 / a.lanes;
  // N == 1: vectors by tokens, then heads; else blocks of tokens, then heads, then tokens
  const int block = blockIdx.x / a.per_heads, first = N == 1 ? (int)blockIdx.x * step : block * N * step;
  const int d = lane * 8;
  const oz2_rows& x = a.x[which];
  float v[N][8];
  int token[N], head[N];
  bool mine[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = first + n * step + (int)threadIdx.x / a.lanes, count = N == 1 ? a.total : (int)a.on.tokens, at = min(i, count - 1);
    mine[n] = i < count && d < a.c.dim;
    token[n] = N == 1 ? at / a.per_heads : at;
    head[n] = N == 1 ? at - token[n] * a.heads : (int)blockIdx.x - block * a.heads;
    if (mine[n]) kv_load8<XT>(x.data, token[n] * x.ld_token + head[n] * x.ld_head + d, v[n]);
  }

  // where they go: the sequence of the workgroup's first token, or one behind it
  const int begin = N == 1 ? first / a.per_heads : first;
  int64_t s = kv_sequence(a.on.sequences, [&](int64_t i) { return a.on.cu[i] <= begin; });
#pragma unroll
  for (int n = 0; n < N; ++n) {
    s = kv_behind(a.on, s, token[n]);
    const KvRange r = kv_range(a.on.cu, s, a.on.tokens);
    const bool packed = mine[n] && token[n] >= r.begin && token[n] < r.end;  // rows behind the last sequence are nobody's
    const int place = kv_held(a.on.lengths, s, a.capacity) - (int)(r.end - token[n]);
    const int at = place / a.per_page;
    int page = -1;
    if (packed && place >= 0) page = a.on.table[s * a.on.ld_table + at];
    const bool goes = page >= 0 && page < a.c.pages;

    // (minimum and maximum keep a NaN)
    float low = v[n][0], high = low;
    if (mine[n]) {
#pragma unroll
      for (int j = 1; j < 8; ++j) low = __builtin_elementwise_minimum(low, v[n][j]), high = __builtin_elementwise_maximum(high, v[n][j]);
    } else low = INFINITY, high = -INFINITY;
    low = over(low, a.lanes, [](float p, float q) { return __builtin_elementwise_minimum(p, q); });
    high = over(high, a.lanes, [](float p, float q) { return __builtin_elementwise_maximum(p, q); });
    // The quotient by 15 and the reciprocal, rounded correctly: what an approximation leaves is exact in an FMA, and once corrected by it is the nearest value
    // (Markstein; neither 15 nor an FP16 value has a significand of ones alone).  Where the range is infinite they are NaNs.
    const float range = high - low, part = range * (1.f / 15.f);
    float fifteenth = fmaf(fmaf(-15.f, part, range), 1.f / 15.f, part);
    asm("" : "+v"(fifteenth));  // (an FP32 value, not an FMA rounded straight to FP16, which differs in one of 20000)
    const _Float16 scale = (_Float16)fifteenth, offset = (_Float16)low;
    const float s32 = (float)scale, o32 = (float)offset, near = __builtin_amdgcn_rcpf(s32);
    const float inverse = s32 == 0.f ? 0.f : fmaf(fmaf(-s32, near, 1.f), near, near);
    unsigned word = 0;
    if (mine[n]) {
      float c[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        c[j] = __builtin_amdgcn_fmed3f(rintf((v[n][j] - o32) * inverse), 0.f, 15.f);  // (of a NaN: 0)
        v[n][j] = fmaf(s32, c[j], o32);
      }
      auto four = [&](int i) { return (unsigned)fmaf(fmaf(c[i + 3], 16.f, c[i + 2]), 256.f, fmaf(c[i + 1], 16.f, c[i])); };
      word = four(0) | four(4) << 16;
    }
    if (goes) {
      const int in = place - at * a.page_size;
      uint8_t* codes = which ? a.c.v_codes : a.c.k_codes;
      *reinterpret_cast<unsigned*>(codes + page * a.c.codes_page + head[n] * a.c.codes_head + (int64_t)in * (a.c.dim / 2) + d / 2) = word;
      if (lane == 0) {
        unsigned* scales = static_cast<unsigned*>(which ? a.c.v_scales : a.c.k_scales);
        scales[page * a.c.scales_page + head[n] * a.c.scales_head + in] = __builtin_bit_cast(uint16_t, scale) | (unsigned)__builtin_bit_cast(uint16_t, offset) << 16;
        if (!which && a.at) a.on.positions[s * a.on.positions_sequence + head[n] * a.on.positions_head + place] = a.at[token[n]];
        if (!which && a.on.weights) a.on.weights[s * a.on.weights_sequence + head[n] * a.on.weights_head + place] = 0.f;
      }
    }
    const oz2_rows& h = a.held[which];
    if (h.data && packed) kv_store8<XT>(h.data, token[n] * h.ld_token + head[n] * h.ld_head + d, v[n]);
  }
}

template <int XT>
hipError_t append(const Append& a, hipStream_t st) {
  const int step = 256 / a.lanes;
  const int64_t once = (a.total + step - 1) / step, blocks = (a.on.tokens + 4 * step - 1) / (4 * step);
  // (four at once where that leaves every compute unit eight workgroups.  27100 tokens of 8 heads of 128 values, us a call one by one and so: BF16 58.6 and 53.7,
  // FP16 55.7 and 52.6, FP32 64.4 and 60.6; with what is held of them written too 71.6 and 72.3, 70.9 and 71.8, 91.7 and 98.3)
  if (once >= 4 * 1024) hipLaunchKernelGGL((kv4_append_kernel<XT, 4>), dim3((unsigned)(blocks * a.heads), 2), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((kv4_append_kernel<XT, 1>), dim3((unsigned)once, 2), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t oz2_launch_kv4_append(const oz2_kv4_cache& cache, const oz2_kv4_sequences& on, const int32_t* at, const oz2_rows& k, const oz2_rows& v,
                                 const oz2_rows* held_k, const oz2_rows* held_v, hipStream_t st) {
  Append a = {cache, on, at, {k, v}, {held_k ? *held_k : oz2_rows{}, held_v ? *held_v : oz2_rows{}}, (int)(on.max_pages * cache.page_size), (int)cache.heads,
              (int)cache.page_size, 1, (int)(on.tokens * cache.heads), fast_div((unsigned)cache.heads), fast_div((unsigned)cache.page_size)};
  while (a.lanes * 8 < cache.dim) a.lanes *= 2;
  return k.type == OZ2_F32 ? append<OZ2_F32>(a, st) : k.type == OZ2_BF16 ? append<OZ2_BF16>(a, st) : append<OZ2_F16>(a, st);
}
