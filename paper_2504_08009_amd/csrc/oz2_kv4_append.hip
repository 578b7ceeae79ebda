// New tokens' keys and values into a cache held in 4 bits (oz2_kv4_append): a vector of dim values becomes dim codes with a scale and an offset.
//
// A vector belongs to the smallest power of two of lanes that have eight values each, which is one word of codes a lane; smallest and largest value are found
// by shuffles.  Bound by the bytes of k and v.
#include "oz2_kv4.h"
#include "oz2_fast_div.h"
#include "oz2_w4_core.h"

namespace {

struct Append {
  oz2_kv4_cache c;
  oz2_kv4_sequences on;
  const int32_t* at;
  oz2_rows x[2], held[2];
  int capacity, heads, page_size, lanes, vectors, total;  // vectors: a workgroup's
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

template <int XT>
__global__ void __launch_bounds__(256) kv4_append_kernel(Append a) {
  const int which = blockIdx.y;  // 0: keys, 1: values
  const int lane = threadIdx.x % a.lanes, first = blockIdx.x * a.vectors;
  const int vector = min(first + (int)threadIdx.x / a.lanes, a.total - 1), token = vector / a.per_heads, head = vector - token * a.heads;
  const int d = lane * 8;
  const oz2_rows& x = a.x[which];
  float v[8];
  const bool mine = first + (int)threadIdx.x / a.lanes < a.total && d < a.c.dim;
  if (mine) kv_load8<XT>(x.data, token * x.ld_token + head * x.ld_head + d, v);

  // where it goes: the sequence of the workgroup's first token, or one behind it
  const int begin = first / a.per_heads;
  int64_t s = kv_sequence(a.on.sequences, [&](int64_t i) { return a.on.cu[i] <= begin; });
  while (s + 1 < a.on.sequences && a.on.cu[s + 1] <= token) ++s;
  const KvRange r = kv_range(a.on.cu, s, a.on.tokens);
  const bool packed = mine && token >= r.begin && token < r.end;  // rows behind the last sequence are nobody's
  const int place = kv_held(a.on.lengths, s, a.capacity) - (int)(r.end - token);
  const int at = place / a.per_page;
  int page = -1;
  if (packed && place >= 0) page = a.on.table[s * a.on.ld_table + at];
  const bool goes = page >= 0 && page < a.c.pages;

  float low = INFINITY, high = -INFINITY, finite = 0.f;
  if (mine) {
#pragma unroll
    for (int j = 0; j < 8; ++j) low = fminf(low, v[j]), high = fmaxf(high, v[j]), finite = fmaf(v[j], 0.f, finite);
  }
  low = over(low, a.lanes, [](float p, float q) { return fminf(p, q); });
  high = over(high, a.lanes, [](float p, float q) { return fmaxf(p, q); });
  finite = over(finite, a.lanes, [](float p, float q) { return p + q; });  // 0, or a NaN where a value is a NaN or an infinity
  const _Float16 scale = (_Float16)((high - low) / 15.f + finite), offset = (_Float16)low;
  const float s32 = (float)scale, o32 = (float)offset, inverse = 1.f / s32;
  unsigned word = 0;
  if (mine) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // (fmaxf and fminf take the other operand for a NaN: a code is 0 .. 15 whatever the value)
      const float c = s32 == 0.f ? 0.f : fminf(fmaxf(rintf((v[j] - o32) * inverse), 0.f), 15.f);
      word |= (unsigned)c << (4 * j);
      v[j] = fmaf(s32, c, o32);
    }
  }
  if (goes) {
    const int in = place - at * a.page_size;
    uint8_t* codes = which ? a.c.v_codes : a.c.k_codes;
    *reinterpret_cast<unsigned*>(codes + page * a.c.codes_page + head * a.c.codes_head + (int64_t)in * (a.c.dim / 2) + d / 2) = word;
    if (lane == 0) {
      unsigned* scales = static_cast<unsigned*>(which ? a.c.v_scales : a.c.k_scales);
      scales[page * a.c.scales_page + head * a.c.scales_head + in] = __builtin_bit_cast(uint16_t, scale) | (unsigned)__builtin_bit_cast(uint16_t, offset) << 16;
      if (!which && a.at) a.on.positions[s * a.on.positions_sequence + head * a.on.positions_head + place] = a.at[token];
      if (!which && a.on.weights) a.on.weights[s * a.on.weights_sequence + head * a.on.weights_head + place] = 0.f;
    }
  }
  const oz2_rows& h = a.held[which];
  if (h.data && packed) kv_store8<XT>(h.data, token * h.ld_token + head * h.ld_head + d, v);
}

}  // namespace

hipError_t oz2_launch_kv4_append(const oz2_kv4_cache& cache, const oz2_kv4_sequences& on, const int32_t* at, const oz2_rows& k, const oz2_rows& v,
                                 const oz2_rows* held_k, const oz2_rows* held_v, hipStream_t st) {
  Append a = {cache, on, at, {k, v}, {held_k ? *held_k : oz2_rows{}, held_v ? *held_v : oz2_rows{}}, (int)(on.max_pages * cache.page_size), (int)cache.heads,
              (int)cache.page_size, 1, 256, (int)(on.tokens * cache.heads), fast_div((unsigned)cache.heads), fast_div((unsigned)cache.page_size)};
  while (a.lanes * 8 < cache.dim) a.lanes *= 2;
  a.vectors = 256 / a.lanes;
  const dim3 grid((unsigned)((a.total + a.vectors - 1) / a.vectors), 2);
  if (k.type == OZ2_F32) hipLaunchKernelGGL(kv4_append_kernel<OZ2_F32>, grid, dim3(256), 0, st, a);
  else if (k.type == OZ2_BF16) hipLaunchKernelGGL(kv4_append_kernel<OZ2_BF16>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(kv4_append_kernel<OZ2_F16>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}
