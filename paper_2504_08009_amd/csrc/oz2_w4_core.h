// What the products with weights held in 4 bits share: how a matrix looks to a launch, how codes become operands, the ends of rows.
//
// A group's sum of (q - z) x is formed from 16-bit floats.  A code is put into the upper mantissa bits of one whose exponent makes it 16 + q
// exactly (one shift, one and-or for two codes; q in the lower bits would be 128 + q, which cancels three more bits), x is taken as it is
// (bf16, f16) or as the three bf16 values that make it up exactly (f32), and
//   sum (q - z) x = sum (16 + q) x - (16 + z) sum x.
// Products of these are exact in FP32, in which everything is summed.  The scale multiplies a group's sum, so that nothing is rounded to
// 16 bits before the result.  The difference cancels: its error is that of sums of (16 + q) |x| and (16 + z) |x|, which in an FP32 result can be several times
// that of a sum of (q - z) x; a 16-bit result does not show it.
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

// threadIdx.x, anew: what follows from it is not kept in registers over the loops around.
__device__ __forceinline__ int w4_thread() {
  int i = threadIdx.x;
  asm volatile("" : "+v"(i));
  return i;
}

constexpr int kW4Block = 128;  // inner indexes that a wave takes at a time: 16 bytes of codes a lane
constexpr float kW4Offset = 16.f;
constexpr float kW4Large = 1e34f;  // where sums of |x| over a few values get there, 31 sum |x| over a group might leave the range of FP32

// 16-bit floats a value of x is made of
template <int XT>
constexpr int w4_parts() { return XT == OZ2_F32 ? 3 : 1; }

// Matrix as a launch sees it: group and scales by blocks of 128.
struct W4Rows {
  const uint8_t* codes;
  const char* scales;
  const uint8_t* zeros;
  int64_t ld_codes, ld_scales, ld_zeros;
  int n, k, group, bytes, full, groups;  // full: whole blocks
  unsigned recip, keep;  // group of block b: the upper half of b recip, recip = ceil(2^32 / blocks of a group), or, where that is one, b
};

// The lane's row of a tile of sixteen, and the registers that a block of it takes.  All loads of a block are made whatever the place: a
// load that a branch may leave out makes the compiler wait for younger ones.
struct W4Lane {
  const uint8_t* codes;
  const char* scales;
  const uint8_t* zeros;
};
template <int SPB>
using W4Words = unsigned __attribute__((ext_vector_type(SPB)));
// Bytes of a block's scales or zero points, of a type that is no wider (else the compiler widens them where the loop turns, and waits
// for them there).
template <int BYTES> struct W4Width { typedef w4_u4 type; };
template <> struct W4Width<8> { typedef W4Words<2> type; };
template <> struct W4Width<4> { typedef unsigned type; };
template <> struct W4Width<2> { typedef unsigned short type; };
template <> struct W4Width<1> { typedef unsigned char type; };
template <int BYTES>
__device__ __forceinline__ typename W4Width<BYTES>::type w4_bytes(const void* p) {
  struct __attribute__((packed, aligned(1))) Any { typename W4Width<BYTES>::type v; };
  return reinterpret_cast<const Any*>(p)->v;
}
template <int BYTES>
__device__ __forceinline__ unsigned w4_word(typename W4Width<BYTES>::type v, int i) {
  if constexpr (BYTES > 4) return v[i];
  else return v;
}
template <int SPB, int ST>
struct W4Regs {
  w4_u4 q;
  typename W4Width<SPB * (ST == OZ2_F32 ? 4 : 2)>::type s;  // as they lie in memory
  typename W4Width<SPB>::type z;  // a byte each
};
template <int SPB>
struct W4Tail {
  w4_u4 q;
  int cut;  // bytes by which q begins early
  W4Words<SPB> s, z;  // one each
};

template <int ST>
__device__ __forceinline__ W4Lane w4_lane(const W4Rows& w, int64_t row) {
  row = row < w.n ? row : w.n - 1;  // rows past the end read the last one; nothing is stored of them
  W4Lane l;
  l.codes = w.codes + row * w.ld_codes + w4_thread() % 64 / 16 * 16;
  l.scales = w.scales + row * w.ld_scales * (ST == OZ2_F32 ? 4 : 2);
  l.zeros = w.zeros + row * w.ld_zeros;
  return l;
}

template <int SPB>
__device__ __forceinline__ int w4_group(const W4Rows& w, int b) {
  if constexpr (SPB > 1) return b * SPB;
  // b below 2^16 and no more blocks in a group than there are blocks: exact, since 2^32 / blocks is exceeded by less than one
  return (int)(__umulhi((unsigned)b, w.recip) + ((unsigned)b & w.keep));
}

// The block behind the whole ones, of rows of at least 16 bytes.  A lane whose bytes are not all there loads the sixteen that end with the
// row, and cuts off later what came early; codes past the end may be anything, since x is 0 there.
template <int SPB, int ST, bool ZEROS>
__device__ __forceinline__ W4Tail<SPB> w4_fetch_tail(const W4Rows& w, const W4Lane& l) {
  W4Tail<SPB> r;
  const int quarter = w4_thread() % 64 / 16;
  const int left = w.bytes - w.full * (kW4Block / 2) - quarter * 16;  // bytes from the lane's first on
  r.cut = left >= 16 || left <= 0 ? 0 : 16 - left;
  r.q = w4_bytes<16>(left > 0 ? l.codes + (int64_t)w.full * (kW4Block / 2) - r.cut : l.codes - quarter * 16);
  const int g = w4_group<SPB>(w, w.full);
  w4_each<SPB>([&](auto i) __attribute__((always_inline)) {
    const int at = min(g + i.value, w.groups - 1);
    if constexpr (ST == OZ2_F32) r.s[i.value] = w4_bytes<4>(l.scales + (int64_t)at * 4);
    else r.s[i.value] = w4_bytes<2>(l.scales + (int64_t)at * 2);
    if constexpr (ZEROS) r.z[i.value] = l.zeros[at];
    else r.z[i.value] = 8u;
  });
  return r;
}

// 16 bytes without the first `cut` (below 16), zeros behind.
__device__ __forceinline__ w4_u4 w4_cut(w4_u4 v, int cut) {
  unsigned long long lo = v[0] | (unsigned long long)v[1] << 32, hi = v[2] | (unsigned long long)v[3] << 32;
  const int bits = 8 * cut;
  if (bits >= 64) lo = hi >> (bits - 64), hi = 0;
  else if (bits) lo = lo >> bits | hi << (64 - bits), hi >>= bits;
  return w4_u4{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
}

__device__ __forceinline__ float w4_decode16(int type, unsigned v) {  // of the lower half
  return type == OZ2_BF16 ? __uint_as_float(v << 16) : (float)__builtin_bit_cast(_Float16, (unsigned short)v);
}
// Eight codes as 16 + q in pairs (0, 4), (1, 5), (2, 6), (3, 7).  The constants come from registers, one of them from a vector register:
// then the and and the or are one instruction, which takes no literals.
template <int XT>
__device__ __forceinline__ void w4_unpack(unsigned w, unsigned out[4]) {
  unsigned m = XT == OZ2_F16 ? 0x03C003C0u : 0x00780078u, c = XT == OZ2_F16 ? 0x4C004C00u : 0x41804180u;
  asm("" : "+s"(m));
  asm("" : "+v"(c));
  if constexpr (XT == OZ2_F16) {
    out[0] = (w << 6 & m) | c, out[1] = (w << 2 & m) | c, out[2] = (w >> 2 & m) | c, out[3] = (w >> 6 & m) | c;
  } else {
    out[0] = (w << 3 & m) | c, out[1] = (w >> 1 & m) | c, out[2] = (w >> 5 & m) | c, out[3] = (w >> 9 & m) | c;
  }
}

// Eight 16-bit floats: their order as that of the pairs above, their sum, and that of their sizes.
__device__ __forceinline__ w4_u4 w4_pairs(w4_u4 v) {
  return w4_u4{__builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[2], v[0], 0x07060302u),
               __builtin_amdgcn_perm(v[3], v[1], 0x05040100u), __builtin_amdgcn_perm(v[3], v[1], 0x07060302u)};
}
typedef __bf16 w4_bf2 __attribute__((ext_vector_type(2)));
typedef _Float16 w4_h2 __attribute__((ext_vector_type(2)));
template <int XT>
__device__ __forceinline__ float w4_dot2(unsigned a, unsigned b, float c) {
  if constexpr (XT == OZ2_F16) return __builtin_amdgcn_fdot2(__builtin_bit_cast(w4_h2, a), __builtin_bit_cast(w4_h2, b), c, false);
  else return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(w4_bf2, a), __builtin_bit_cast(w4_bf2, b), c, false);
}
template <int XT>
__device__ __forceinline__ void w4_sums(w4_u4 v, float& s, float& a) {
  constexpr unsigned one = XT == OZ2_F16 ? 0x3C003C00u : 0x3F803F80u;
#pragma unroll
  for (int i = 0; i < 4; ++i) s = w4_dot2<XT>(v[i], one, s), a = w4_dot2<XT>(v[i] & 0x7FFF7FFFu, one, a);
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

// x in LDS.  A token's values lie in rows of `pitch` bytes for each of its parts, eight at a time in the order of w4_unpack's pairs.  Row a of the
// matrix cores' tile is token a / 4 + 4 (a % 4), so that with few tokens only the first result registers of a lane count (RT: 1 or 4
// for up to 4 or 16 tokens).
// Row a without a token reads the last one's, and nobody looks at its results.  (The rows of a quarter that read one place together cost nothing.)
template <int PARTS>
__device__ __forceinline__ int w4_row_of_x(int a, int tokens, int pitch) {
  return min(a / 4 + 4 * (a % 4), tokens - 1) * PARTS * pitch;
}

// Value of the lane across in a pair, four, eight or sixteen lanes whose halves hold one value each (a pair: its two lanes).
template <int STEP>
__device__ __forceinline__ float w4_partner(float v) {
  constexpr int ctrl = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x141 : 0x140;  // quad permutations, mirrors of 8 and 16 lanes
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), ctrl, 0xF, 0xF, true));
}
#endif
#endif
