// Rows held in 4 bits times one or two vectors, by the vector units: a lane holds 32 neighbouring values of x in registers and meets the 16
// bytes of codes that go with them, row after row.  Nothing goes through LDS, four lanes read 64 bytes in a row, and a lane's codes lie in
// one group, so that its sum needs one scale.
#ifndef OZ2_W4_VECTOR_H
#define OZ2_W4_VECTOR_H

#include "oz2_w4_core.h"

#ifdef __HIPCC__

constexpr int kW4Unit = 32;                 // inner indexes of a lane
constexpr int kW4Span = 64 * kW4Unit;       // of a wave

typedef __bf16 w4_bf2 __attribute__((ext_vector_type(2)));
typedef _Float16 w4_h2 __attribute__((ext_vector_type(2)));

// A lane's 32 values of x (pairs in the order of w4_unpack, or FP32), their sum, and where it finds the codes and scales of a row.
template <int XT>
struct W4X {
  unsigned v[XT == OZ2_F32 ? 32 : 16];
  float sum;
};
struct W4Place {
  int codes, cut;  // bytes from the row's start; bytes that come early (the lane in which the row ends loads the last 16)
  int group;
};

__device__ __forceinline__ W4Place w4_place(const W4Rows& w, int unit) {
  const int left = w.bytes - unit * (kW4Unit / 2);
  W4Place p = {0, 0, 0};  // (past the end: the row's first bytes, whose x is 0)
  if (left > 0) {
    p.cut = left < 16 ? 16 - left : 0;
    p.codes = unit * (kW4Unit / 2) - p.cut;
    p.group = unit / (w.group / kW4Unit);
  }
  return p;
}

template <int XT>
__device__ __forceinline__ void w4_load_x(const char* x, int k, int unit, w4_u4 raw[XT == OZ2_F32 ? 8 : 4]) {
  constexpr int size = XT == OZ2_F32 ? 4 : 2, per = 16 / size;
#pragma unroll
  for (int j = 0; j < kW4Unit / per; ++j) raw[j] = w4_bytes<16>(x + (int64_t)min(unit * kW4Unit + j * per, k - per) * size);
}
template <int XT>
__device__ __forceinline__ W4X<XT> w4_keep_x(int k, int unit, w4_u4 raw[XT == OZ2_F32 ? 8 : 4], bool& plain) {
  constexpr int size = XT == OZ2_F32 ? 4 : 2, per = 16 / size;
  W4X<XT> x;
  if ((unit + 1) * kW4Unit > k) {
#pragma unroll
    for (int j = 0; j < kW4Unit / per; ++j) {
      const int there = k - (unit * kW4Unit + j * per);
      raw[j] = there <= 0 ? w4_u4{0, 0, 0, 0} : there < per ? w4_cut(raw[j], (per - there) * size) : raw[j];
    }
  }
  float s = 0.f, a = 0.f;
#pragma unroll
  for (int j = 0; j < kW4Unit / per; ++j) {
    if constexpr (XT == OZ2_F32) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x.v[4 * j + e] = raw[j][e];
        s += __uint_as_float(raw[j][e]), a += fabsf(__uint_as_float(raw[j][e]));
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float lo = w4_decode16(XT, raw[j][e] & 0xFFFFu), hi = w4_decode16(XT, raw[j][e] >> 16);
        s += lo + hi, a += fabsf(lo) + fabsf(hi);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // (0, 4), (1, 5), (2, 6), (3, 7)
        const unsigned lo = raw[j][e / 2], hi = raw[j][2 + e / 2];
        x.v[4 * j + e] = e % 2 ? (lo >> 16) | (hi & 0xFFFF0000u) : (lo & 0xFFFFu) | hi << 16;
      }
    }
  }
  x.sum = s;
  plain |= !(a < kW4Large);
  return x;
}

// sum of (16 + q) x (16-bit x) or q x (FP32 x) over the lane's codes, for T vectors at once
template <int XT, int T, int NC>
__device__ __forceinline__ void w4_dot(w4_u4 codes, const W4X<XT> (&x)[T][NC], int c, float out[T]) {
  float a[T][2];
#pragma unroll
  for (int t = 0; t < T; ++t) a[t][0] = a[t][1] = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (XT == OZ2_F32) {
      const unsigned even = codes[j] & 0x0F0F0F0Fu, odd = codes[j] >> 4 & 0x0F0F0F0Fu;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float q = (float)(even >> (8 * e) & 255u), r = (float)(odd >> (8 * e) & 255u);
#pragma unroll
        for (int t = 0; t < T; ++t) {
          a[t][0] = fmaf(q, __uint_as_float(x[t][c].v[8 * j + 2 * e]), a[t][0]);
          a[t][1] = fmaf(r, __uint_as_float(x[t][c].v[8 * j + 2 * e + 1]), a[t][1]);
        }
      }
    } else {
      unsigned b[4];
      w4_unpack<XT>(codes[j], b);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < T; ++t) {
          if constexpr (XT == OZ2_BF16)
            a[t][e % 2] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(w4_bf2, b[e]), __builtin_bit_cast(w4_bf2, x[t][c].v[4 * j + e]), a[t][e % 2], false);
          else
            a[t][e % 2] = __builtin_amdgcn_fdot2(__builtin_bit_cast(w4_h2, b[e]), __builtin_bit_cast(w4_h2, x[t][c].v[4 * j + e]), a[t][e % 2], false);
        }
    }
  }
#pragma unroll
  for (int t = 0; t < T; ++t) out[t] = a[t][0] + a[t][1];
}

// The same for the row, straight from memory, with s (q - z) x one by one: for x with infinities, NaNs or values near the end of the range.
template <int XT, int ST, bool ZEROS>
__device__ __forceinline__ float w4_unit_plain(const W4Rows& w, const uint8_t* codes, const char* scales, const uint8_t* zeros, int64_t row, const char* x,
                                               int unit) {
  const int end = min((unit + 1) * kW4Unit, w.k), g = unit / (w.group / kW4Unit);
  float sum = 0.f;
#pragma unroll 1
  for (int i = unit * kW4Unit; i < end; ++i) {
    const int q = codes[row * w.ld_codes + i / 2] >> (i % 2 * 4) & 15;
    sum = fmaf(w4_load(ST, scales, row * w.ld_scales + g) * (float)(q - (ZEROS ? (int)zeros[row * w.ld_zeros + g] : 8)), w4_load(XT, x, i), sum);
  }
  return sum;
}

// Sums of four values over the wave: lane l gets that of value l / 16.
__device__ __forceinline__ float w4_sum4(float a, float b, float c, float d) {
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  auto pair32 = [](float p, float q) {
    const u2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(p), __float_as_uint(q), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  };
  const float p = pair32(a, c), q = pair32(b, d);
  const u2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(p), __float_as_uint(q), false, false);
  float v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  v += w4_partner<0>(v), v += w4_partner<1>(v), v += w4_partner<2>(v), v += w4_partner<3>(v);
  return v;
}

// Four rows (from `row`, those past the end repeat the last) times T vectors, the inner indexes of this wave's NC spans; x as kept.
// All loads first: R * NC of 16 bytes a lane are in flight.
template <int XT, int T, int NC, int ST, bool ZEROS>
struct W4Rows4 {
  W4Regs<1, ST> r[4][NC];

  __device__ __forceinline__ void fetch(const W4Rows& w, const uint8_t* codes, const char* scales, const uint8_t* zeros, int row, const W4Place (&at)[NC]) {
    constexpr int size = ST == OZ2_F32 ? 4 : 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t n = min(row + i, w.n - 1);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        r[i][c].q = w4_bytes<16>(codes + n * w.ld_codes + at[c].codes);
        r[i][c].s = w4_bytes<size>(scales + n * w.ld_scales * size + at[c].group * size);
        if constexpr (ZEROS) r[i][c].z = zeros[n * w.ld_zeros + at[c].group];
      }
    }
  }

  // sum[i][t] of the lane
  __device__ __forceinline__ void multiply(const W4Place (&at)[NC], const W4X<XT> (&x)[T][NC], const bool (&ragged)[NC], float (&sum)[4][T]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int t = 0; t < T; ++t) sum[i][t] = 0.f;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        w4_u4 q = r[i][c].q;
        if (ragged[c]) q = w4_cut(q, at[c].cut);
        float s, z = 8.f;
        if constexpr (ST == OZ2_F32) s = __uint_as_float(r[i][c].s);
        else s = w4_decode16(ST, r[i][c].s);
        if constexpr (ZEROS) z = (float)r[i][c].z;
        float p[T];
        w4_dot<XT, T, NC>(q, x, c, p);
#pragma unroll
        for (int t = 0; t < T; ++t) sum[i][t] = fmaf(s, fmaf(-(XT == OZ2_F32 ? z : z + kW4Offset), x[t][c].sum, p[t]), sum[i][t]);
      }
    }
  }

  __device__ __forceinline__ void multiply_plain(const W4Rows& w, const uint8_t* codes, const char* scales, const uint8_t* zeros, int row, const char* x,
                                                 int64_t ldx, int unit, float (&sum)[4][T]) {
#pragma unroll 1
    for (int j = 0; j < 4 * T; ++j) {
      float v = 0.f;
#pragma unroll 1
      for (int c = 0; c < NC; ++c)
        v += w4_unit_plain<XT, ST, ZEROS>(w, codes, scales, zeros, min(row + j / T, w.n - 1), x + j % T * ldx * (XT == OZ2_F32 ? 4 : 2), unit + 64 * c);
      w4_each<4 * T>([&](auto i) __attribute__((always_inline)) {
        if (j == i.value) sum[i.value / T][i.value % T] = v;
      });
    }
  }
};

#endif
#endif
