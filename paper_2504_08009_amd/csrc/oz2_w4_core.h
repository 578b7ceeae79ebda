// What the products with weights held in 4 bits share: sixteen rows of a matrix times up to sixteen vectors, by one wave.
//
// A group's sum of (q - z) x is formed on the matrix cores.  A code is put into the upper mantissa bits of a 16-bit float whose exponent
// makes it 16 + q exactly (one shift, one and-or for two codes; q in the lower bits would be 128 + q, which cancels three more bits), x
// is taken as it is (bf16, f16) or as the three bf16 values that make it up exactly (f32), and
//   sum (q - z) x = sum (16 + q) x - (16 + z) sum x
// with the sums of x per group formed once, where x is brought into LDS.  Products of these are exact in FP32, in which everything is summed.
// The scale multiplies a group's sum, so that nothing is rounded to 16 bits before the result.
#ifndef OZ2_W4_CORE_H
#define OZ2_W4_CORE_H

#include "oz2_w4.h"

#ifdef __HIPCC__

typedef unsigned w4_u4 __attribute__((ext_vector_type(4)));
typedef float w4_f4 __attribute__((ext_vector_type(4)));
typedef __bf16 w4_bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 w4_h8 __attribute__((ext_vector_type(8)));

// f(0), f(1), ..., f(N - 1) with constants: for loops over arrays of registers, which must not be indexed by a variable.
template <int I>
struct W4Index { static constexpr int value = I; };
template <int N, class F>
__device__ __forceinline__ void w4_each(F f) {
  if constexpr (N > 0) {
    w4_each<N - 1>(f);
    f(W4Index<N - 1>{});
  }
}

struct __attribute__((packed, aligned(1))) W4Bytes16 { unsigned v[4]; };
struct __attribute__((packed, aligned(1))) W4Bytes8 { unsigned v[2]; };
struct __attribute__((packed, aligned(1))) W4Bytes4 { unsigned v; };
struct __attribute__((packed, aligned(1))) W4Bytes2 { unsigned short v; };

constexpr int kW4Block = 128;  // inner indexes that a wave takes at a time: 16 bytes of codes a lane
constexpr float kW4Offset = 16.f;
constexpr float kW4Large = 1e36f;  // sums of |x| over a group from here on are not trusted to 31 sum |x| in FP32

// 16-bit floats a value of x is made of
template <int XT>
constexpr int w4_parts() { return XT == OZ2_F32 ? 3 : 1; }

// Matrix as a launch sees it: group and scales by blocks of 128.
struct W4Rows {
  const uint8_t* codes;
  const char* scales;
  const uint8_t* zeros;
  int64_t ld_codes, ld_scales, ld_zeros;
  int n, k, bytes, blocks, groups;
  int shift, per_group;  // blocks of a group (where that is 128 or more): 1 << shift, or per_group where shift < 0
  int scale_type;
};

// The lane's row of a tile of sixteen, and the registers that a block of it takes.
struct W4Lane {
  const uint8_t* codes;
  const char* scales;
  const uint8_t* zeros;
};
template <int SPB>
struct W4Regs {
  w4_u4 q;
  unsigned __attribute__((ext_vector_type(SPB))) s;
  unsigned z;
};

__device__ __forceinline__ W4Lane w4_lane(const W4Rows& w, int64_t row) {
  row = row < w.n ? row : w.n - 1;  // rows past the end read the last one; nothing is stored of them
  W4Lane l;
  const int size = w.scale_type == OZ2_F32 ? 4 : 2;
  l.codes = w.codes + row * w.ld_codes + (threadIdx.x % 64 / 16) * 16;
  l.scales = w.scales + row * w.ld_scales * size;
  l.zeros = w.zeros ? w.zeros + row * w.ld_zeros : nullptr;
  return l;
}

// Block b of the row: 16 bytes of codes for this lane, and the scales and zero points of its segments (a group, or 128 of one).
// (Values are returned and assigned whole: stores into parts of an array from different branches would put it into memory.)
__device__ __forceinline__ w4_u4 w4_fetch_codes(const W4Rows& w, const W4Lane& l, int b) {
  const uint8_t* p = l.codes + (int64_t)b * (kW4Block / 2);
  if ((b + 1) * (kW4Block / 2) <= w.bytes) {
    const W4Bytes16 c = *reinterpret_cast<const W4Bytes16*>(p);
    return w4_u4{c.v[0], c.v[1], c.v[2], c.v[3]};
  }
  // the row's last block: no byte past its end
  const int left = w.bytes - b * (kW4Block / 2) - (threadIdx.x % 64 / 16) * 16;
  auto word = [&](int i) {
    unsigned v = 0;
#pragma unroll
    for (int j = i; j < i + 4; ++j)
      if (j < left) v |= (unsigned)p[j] << (8 * (j - i));
    return v;
  };
  return w4_u4{word(0), word(4), word(8), word(12)};
}

// As they lie in memory: a word each (f32), or two to a word.
template <int SPB>
using W4Scales = unsigned __attribute__((ext_vector_type(SPB)));
template <int SPB>
__device__ __forceinline__ W4Scales<SPB> w4_fetch_scales(const W4Rows& w, const W4Lane& l, int g) {
  auto wide = [&](int i) { return reinterpret_cast<const W4Bytes4*>(l.scales + (int64_t)(g + i) * 4)->v; };
  auto narrow = [&](int i) { return (unsigned)reinterpret_cast<const W4Bytes2*>(l.scales + (int64_t)(g + i) * 2)->v; };
  if constexpr (SPB == 1) {
    return w.scale_type == OZ2_F32 ? wide(0) : narrow(0);
  } else {
    const bool whole = g + SPB <= w.groups;
    if (w.scale_type == OZ2_F32) {
      if constexpr (SPB == 2) {
        if (whole) { const W4Bytes8 c = *reinterpret_cast<const W4Bytes8*>(l.scales + (int64_t)g * 4); return W4Scales<2>{c.v[0], c.v[1]}; }
        return W4Scales<2>{wide(0), 0u};
      } else {
        if (whole) { const W4Bytes16 c = *reinterpret_cast<const W4Bytes16*>(l.scales + (int64_t)g * 4); return W4Scales<4>{c.v[0], c.v[1], c.v[2], c.v[3]}; }
        const int last = w.groups - 1 - g;  // below 3; segments past the last group get a scale of 0
        return W4Scales<4>{wide(0), last > 0 ? wide(1) : 0u, last > 1 ? wide(2) : 0u, 0u};
      }
    }
    if constexpr (SPB == 2) {
      return W4Scales<2>{whole ? reinterpret_cast<const W4Bytes4*>(l.scales + (int64_t)g * 2)->v : narrow(0), 0u};
    } else {
      if (whole) { const W4Bytes8 c = *reinterpret_cast<const W4Bytes8*>(l.scales + (int64_t)g * 2); return W4Scales<4>{c.v[0], c.v[1], 0u, 0u}; }
      const int last = w.groups - 1 - g;
      return W4Scales<4>{narrow(0) | (last > 0 ? narrow(1) << 16 : 0u), last > 1 ? narrow(2) : 0u, 0u, 0u};
    }
  }
}

// A byte each.
template <int SPB>
__device__ __forceinline__ unsigned w4_fetch_zeros(const W4Rows& w, const W4Lane& l, int g) {
  if (!w.zeros) return 0x08080808u;
  const uint8_t* p = l.zeros + g;
  if constexpr (SPB == 1) return p[0];
  if constexpr (SPB == 2) return g + SPB <= w.groups ? reinterpret_cast<const W4Bytes2*>(p)->v : p[0];
  if (g + SPB <= w.groups) return reinterpret_cast<const W4Bytes4*>(p)->v;
  const int last = w.groups - 1 - g;
  return p[0] | (last > 0 ? (unsigned)p[1] << 8 : 0u) | (last > 1 ? (unsigned)p[2] << 16 : 0u);
}

template <int SPB>
__device__ __forceinline__ W4Regs<SPB> w4_fetch(const W4Rows& w, const W4Lane& l, int b) {
  int g;
  if constexpr (SPB > 1) g = b * SPB;
  else g = w.shift >= 0 ? b >> w.shift : b / w.per_group;
  W4Regs<SPB> r;
  r.q = w4_fetch_codes(w, l, b);
  r.s = w4_fetch_scales<SPB>(w, l, g);
  r.z = w4_fetch_zeros<SPB>(w, l, g);
  return r;
}

__device__ __forceinline__ float w4_decode16(int type, unsigned v) {  // of the lower half
  return type == OZ2_BF16 ? __uint_as_float(v << 16) : (float)__builtin_bit_cast(_Float16, (unsigned short)v);
}
template <int SPB>
__device__ __forceinline__ float w4_scale(int type, const W4Regs<SPB>& r, int seg) {
  return type == OZ2_F32 ? __uint_as_float(r.s[seg]) : w4_decode16(type, r.s[seg / 2] >> (seg % 2 * 16));
}

// Eight codes as 16 + q in pairs (0, 4), (1, 5), (2, 6), (3, 7).
template <int XT>
__device__ __forceinline__ void w4_unpack(unsigned w, unsigned out[4]) {
  if constexpr (XT == OZ2_F16) {
    constexpr unsigned m = 0x03C003C0u, c = 0x4C004C00u;
    out[0] = (w << 6 & m) | c, out[1] = (w << 2 & m) | c, out[2] = (w >> 2 & m) | c, out[3] = (w >> 6 & m) | c;
  } else {
    constexpr unsigned m = 0x00780078u, c = 0x41804180u;
    out[0] = (w << 3 & m) | c, out[1] = (w >> 1 & m) | c, out[2] = (w >> 5 & m) | c, out[3] = (w >> 9 & m) | c;
  }
}

template <int XT>
__device__ __forceinline__ w4_f4 w4_mfma(uint4 x, const unsigned q[4], w4_f4 acc) {
  const uint4 b = make_uint4(q[0], q[1], q[2], q[3]);
  if constexpr (XT == OZ2_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(w4_h8, x), __builtin_bit_cast(w4_h8, b), acc, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(w4_bf8, x), __builtin_bit_cast(w4_bf8, b), acc, 0, 0, 0);
}

// Words of four lanes (one in each quarter of the wave) that hold 32 consecutive codes each are exchanged so that the four words of
// register j belong to one segment: nothing to do where a segment is the whole block.
template <int SPB>
__device__ __forceinline__ w4_u4 w4_exchange(w4_u4 q) {
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  if constexpr (SPB >= 2) {
    const u2 a = __builtin_amdgcn_permlane32_swap(q[0], q[2], false, false), b = __builtin_amdgcn_permlane32_swap(q[1], q[3], false, false);
    q = w4_u4{a[0], b[0], a[1], b[1]};
  }
  if constexpr (SPB == 4) {
    const u2 a = __builtin_amdgcn_permlane16_swap(q[0], q[1], false, false), b = __builtin_amdgcn_permlane16_swap(q[2], q[3], false, false);
    q = w4_u4{a[0], a[1], b[0], b[1]};
  }
  return q;
}
// Register of the j-th product of a block, and the inner index (from the block's start) at which a lane of that quarter stands then.
template <int SPB>
__device__ __forceinline__ constexpr int w4_register(int j) { return SPB == 2 ? (j % 2) + 2 * (j / 2) : j; }
template <int SPB>
__device__ __forceinline__ int w4_inner(int j, int quarter) {
  if constexpr (SPB == 1) return 32 * quarter + 8 * j;
  else if constexpr (SPB == 2) return 64 * (j / 2) + 32 * (quarter % 2) + 16 * (quarter / 2) + 8 * (j % 2);
  else return 32 * j + 8 * quarter;
}

// x in LDS.  A token's values lie in rows of `pitch` bytes for each of its parts, eight at a time in the order of w4_unpack's pairs; the sums
// over segments lie by segment, then by token.  Row a of the matrix cores' tile is token a / 4 + 4 (a % 4), so that with
// few tokens only the first result registers of a lane count (RT: 1, 2 or 4 for up to 4, 8 or 16 tokens).
template <int RT>
__device__ __forceinline__ int w4_token(int a) { return a / 4 + 4 * (a % 4); }

// One block: the lane's sums (tokens quarter + 4 r, its row) grow by  scale ((16 + q) x - (16 + z) x).
// x: the lane's token at the block's start, part p at + p part_bytes; sums: of the block's first segment.
template <int XT, int SPB, int RT>
__device__ __forceinline__ void w4_block(const W4Rows& w, const W4Regs<SPB>& r, const char* x, int part_bytes, const float* sums, float* sum) {
  const int quarter = threadIdx.x % 64 / 16;
  const w4_u4 q = w4_exchange<SPB>(r.q);
  w4_each<SPB>([&](auto index) __attribute__((always_inline)) {
    constexpr int seg = index.value;
    w4_f4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4 / SPB; ++i) {
      const int j = seg * (4 / SPB) + i;
      unsigned b[4];
      w4_unpack<XT>(q[w4_register<SPB>(j)], b);
#pragma unroll
      for (int p = 0; p < w4_parts<XT>(); ++p)
        acc = w4_mfma<XT>(*reinterpret_cast<const uint4*>(x + p * part_bytes + 2 * w4_inner<SPB>(j, quarter)), b, acc);
    }
    const float s = w4_scale<SPB>(w.scale_type, r, seg);
    const float z = kW4Offset + (float)(r.z >> (8 * seg) & 255u);
#pragma unroll
    for (int i = 0; i < RT; ++i) sum[i] = fmaf(s, fmaf(-z, sums[(seg * 4 + quarter) * RT + i], acc[i]), sum[i]);
  });
}

// The same by the formula itself, code by code: for blocks whose x has infinities, NaNs, or values near the end of the range.
template <int SPB, int RT, class X>
__device__ __forceinline__ void w4_block_plain(const W4Rows& w, const W4Lane& l, int b, X value, float* sum) {
  const uint8_t* codes = l.codes - (threadIdx.x % 64 / 16) * 16;
  const int end = min(w.k, (b + 1) * kW4Block);
#pragma unroll 1
  for (int i = b * kW4Block; i < end; ++i) {
    const int q = codes[i / 2] >> (i % 2 * 4) & 15;
    int g;
    if (SPB > 1) g = i / (kW4Block / SPB);
    else g = w.shift >= 0 ? b >> w.shift : b / w.per_group;
    const float s = w4_load(w.scale_type, l.scales, g);
    const float v = s * (float)(q - (w.zeros ? (int)l.zeros[g] : 8));
#pragma unroll
    for (int r = 0; r < RT; ++r) sum[r] = fmaf(v, value(r, i), sum[r]);
  }
}

// Brings inner indexes [first, first + length) of `tokens` vectors into LDS (zeros past k); length is a multiple of 128.  Returns
// whether what this thread saw calls for w4_block_plain.  row(token): element offset of the vector.
template <int XT, int SPB, int RT, class Row>
__device__ __forceinline__ bool w4_stage(const void* x, Row row, int tokens, int k, int first, int length, char* lds, int pitch, float* sums,
                                         int threads) {
  constexpr int SEG = kW4Block / SPB, P = w4_parts<XT>();
  bool plain = false;
  const int eights = length / 8;
  for (int i = threadIdx.x; i < tokens * eights; i += threads) {
    const int t = i / eights, at = (i - t * eights) * 8, l = first + at;
    float v[8];
    unsigned h[P][8];
    if constexpr (XT == OZ2_F32) {
      const float* p = static_cast<const float*>(x) + row(t) + l;
      if (l + 8 <= k) {
        const W4Bytes16 a = *reinterpret_cast<const W4Bytes16*>(p), b = *reinterpret_cast<const W4Bytes16*>(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(a.v[e]), v[e + 4] = __uint_as_float(b.v[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = l + e < k ? p[e] : 0.f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {  // cut, not rounded: each part takes the next eight bits, and none can overflow
        float rest = v[e];
#pragma unroll
        for (int c = 0; c < 3; ++c) {
          h[c][e] = __float_as_uint(rest) >> 16;
          rest -= __uint_as_float(h[c][e] << 16);
        }
      }
    } else {
      const uint16_t* p = static_cast<const uint16_t*>(x) + row(t) + l;
      if (l + 8 <= k) {
        const W4Bytes16 a = *reinterpret_cast<const W4Bytes16*>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[0][e] = a.v[e / 2] >> (e % 2 * 16) & 0xFFFFu;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[0][e] = l + e < k ? p[e] : 0u;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = w4_decode16(XT, h[0][e]);
    }
#pragma unroll
    for (int c = 0; c < P; ++c)
      *reinterpret_cast<uint4*>(lds + (t * P + c) * pitch + 2 * at) =
          make_uint4(h[c][0] | h[c][4] << 16, h[c][1] | h[c][5] << 16, h[c][2] | h[c][6] << 16, h[c][3] | h[c][7] << 16);
    float s = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    float a = ((fabsf(v[0]) + fabsf(v[1])) + (fabsf(v[2]) + fabsf(v[3]))) + ((fabsf(v[4]) + fabsf(v[5])) + (fabsf(v[6]) + fabsf(v[7])));
    // the threads of a segment are neighbours, and all of them are here: `eights` is a multiple of 16
#pragma unroll
    for (int d = 1; d < SEG / 8; d *= 2) s += __shfl_xor(s, d), a += __shfl_xor(a, d);
    plain |= !(a < kW4Large);
    if (at % SEG == 0) sums[(at / SEG * 4 + t % 4) * RT + t / 4] = s;
  }
  return plain;
}

#endif
#endif
