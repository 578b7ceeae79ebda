// Attention over prompts and over caches held in 4 bits: launchers, and what the kernels share.
#ifndef OZ2_KV4_H
#define OZ2_KV4_H

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/oz2.h"

// Launchers; arguments as checked by the entry points.
hipError_t oz2_launch_attention(int64_t tokens, int64_t sequences, const int32_t* cu, int64_t heads, int64_t kv_heads, int64_t dim, float scale, int causal,
                                const oz2_rows& q, const oz2_rows& k, const oz2_rows& v, const oz2_rows& out, hipStream_t st);
hipError_t oz2_launch_kv4_append(const oz2_kv4_cache& cache, const oz2_kv4_sequences& on, const int32_t* at, const oz2_rows& k, const oz2_rows& v,
                                 const oz2_rows* held_k, const oz2_rows* held_v, hipStream_t st);
size_t oz2_kv4_attention_space(const oz2_kv4_cache& cache, int64_t sequences, int64_t max_pages, int64_t tokens, int64_t heads, int weights);
hipError_t oz2_launch_kv4_attention(const oz2_kv4_cache& cache, const oz2_kv4_sequences& on, int64_t heads, float scale, const oz2_rows& q,
                                    const oz2_rows& out, char* ws, hipStream_t st);
size_t oz2_kv4_evict_space(const oz2_kv4_cache& cache, int64_t sequences, int64_t max_pages, int64_t keep);
hipError_t oz2_launch_kv4_evict(const oz2_kv4_cache& cache, const oz2_kv4_sequences& on, int64_t keep, int64_t recent, const oz2_kv4_kept& to, char* ws,
                                hipStream_t st);

#ifdef __HIPCC__
#include "oz2_w4.h"

// Softmax weights are exp2(score scale2 - m), one FMA: m is a row's largest product, rounded, and what its rounding left is part of every weight alike.  From 2^31 on that
// would be 2^128 of them or none.  So a product beyond kLarge is formed with the power of two above scale2 instead, which leaves nothing: m is then a function of the score
// that still rises with it, and differences count up to twice, where neighbouring FP32 numbers are 4 apart and more.
constexpr float kLarge = 0x1p25f, kNoScore = -3.402823466e38f;  // (and the m of a row without a score: no product is below it)
__device__ __forceinline__ float kv_power_above(float x) { return __uint_as_float((__float_as_uint(x) + 0x7fffff) & 0x7f800000); }
__device__ __forceinline__ float kv_scale_of(float score, float scale2) { return fabsf(score * scale2) > kLarge ? kv_power_above(scale2) : scale2; }

// Rows of sequence s among `tokens` packed ones, and how many places it holds: whatever cu and lengths say, within what there is.
struct KvRange { int64_t begin, end; };
__device__ __forceinline__ KvRange kv_range(const int32_t* cu, int64_t s, int64_t tokens) {
  const int64_t a = cu[s], b = cu[s + 1];
  const int64_t begin = a < 0 ? 0 : a < tokens ? a : tokens;
  return {begin, b < begin ? begin : b < tokens ? b : tokens};
}
__device__ __forceinline__ int kv_held(const int32_t* lengths, int64_t s, int capacity) {
  const int n = lengths[s];
  return n < 0 ? 0 : n < capacity ? n : capacity;
}

// The last of `sequences` that has begun, where begun(i) holds up to one and for none behind it (begun(0) is not asked).  Same arguments in all lanes, which ask
// for 64 sequences at a time.
template <class Begun>
__device__ __forceinline__ int64_t kv_sequence(int64_t sequences, Begun begun) {
  int64_t first = 0, n = sequences;
  while (n > 1) {
    const int64_t step = (n + 63) / 64, i = (threadIdx.x % 64 + 1) * step;
    const int64_t k = __popcll(__ballot(i < n && begun(first + i)));
    first += k * step;
    n = n - k * step < step ? n - k * step : step;
  }
  return first;
}

// The last sequence from s on that begins at or before a token: mostly s, so in strides that double, then halve.
__device__ __forceinline__ int64_t kv_behind(const oz2_kv4_sequences& on, int64_t s, int64_t token) {
  int64_t stride = 1;
  for (; s + stride < on.sequences && on.cu[s + stride] <= token; stride *= 2) s += stride;
  for (; stride > 1;) {
    stride /= 2;
    if (s + stride < on.sequences && on.cu[s + stride] <= token) s += stride;
  }
  return s;
}

// Eight values beside each other of a row, in FP32.
template <int XT>
__device__ __forceinline__ void kv_load8(const void* p, int64_t i, float (&x)[8]) {
  if constexpr (XT == OZ2_F32) {
    struct __attribute__((packed, aligned(4))) Eight { float v[8]; };
    const Eight e = *reinterpret_cast<const Eight*>(static_cast<const float*>(p) + i);
    for (int j = 0; j < 8; ++j) x[j] = e.v[j];
  } else {
    struct __attribute__((packed, aligned(2))) Eight { unsigned v[4]; };
    const Eight e = *reinterpret_cast<const Eight*>(static_cast<const uint16_t*>(p) + i);
    for (int j = 0; j < 4; ++j) {
      if constexpr (XT == OZ2_BF16) {
        x[2 * j] = __uint_as_float(e.v[j] << 16);
        x[2 * j + 1] = __uint_as_float(e.v[j] & 0xffff0000u);
      } else {
        x[2 * j] = (float)__builtin_bit_cast(_Float16, (uint16_t)e.v[j]);
        x[2 * j + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(e.v[j] >> 16));
      }
    }
  }
}
template <int XT>
__device__ __forceinline__ void kv_store8(void* p, int64_t i, const float (&x)[8]) {
  if constexpr (XT == OZ2_F32) {
    struct __attribute__((packed, aligned(4))) Eight { float v[8]; };
    Eight e;
    for (int j = 0; j < 8; ++j) e.v[j] = x[j];
    *reinterpret_cast<Eight*>(static_cast<float*>(p) + i) = e;
  } else {
    struct __attribute__((packed, aligned(2))) Eight { unsigned v[4]; };
    Eight e;
    for (int j = 0; j < 4; ++j) {
      uint16_t a, b;
      if constexpr (XT == OZ2_BF16) {
        a = __builtin_bit_cast(uint16_t, (__bf16)x[2 * j]), b = __builtin_bit_cast(uint16_t, (__bf16)x[2 * j + 1]);
      } else {
        a = __builtin_bit_cast(uint16_t, (_Float16)x[2 * j]), b = __builtin_bit_cast(uint16_t, (_Float16)x[2 * j + 1]);
      }
      e.v[j] = a | (unsigned)b << 16;
    }
    *reinterpret_cast<Eight*>(static_cast<uint16_t*>(p) + i) = e;
  }
}
#endif

#endif
