// Rows held in 4 bits times one or two vectors, by the vector units: a lane holds 32 neighbouring values of x in registers and meets the 16
// bytes of codes that go with them, row after row.  Nothing goes through LDS, four lanes read 64 bytes in a row, and a lane's codes lie in
// one group, so that its sum needs one scale.  The sum of (q - z) x is that of (16 + q) x less (16 + z) times the sum of x (FP32 x: of q x less z times it),
// which the lane forms once.
//
// Bound by reading the codes: 65536 x 8192 with one vector takes 53 us, 5.7 TB/s of the 5.9 that reading alone reaches.  Smaller products take
// a launch's time and one trip to memory: 4096 x 4096 4.8 us for 8.7 MB, 16384 x 4096 in half precision 9.4 us for 37 MB.
#ifndef OZ2_W4_VECTOR_H
#define OZ2_W4_VECTOR_H

#include "oz2_w4_core.h"

#ifdef __HIPCC__

constexpr int kW4Unit = 32;                 // inner indexes of a lane
constexpr int kW4Span = 64 * kW4Unit;       // of a wave

// A lane's 32 values of x (pairs in the order of w4_unpack, or FP32), their sum, and where it finds the codes and scales of a row.
template <int XT>
struct W4X {
  unsigned v[XT == OZ2_F32 ? 32 : 16];
  float sum;
};
// (Unsigned: the offset of a load from a row's start, which is in scalar registers.)
struct W4Place {
  unsigned codes, group;  // bytes from the row's start; of the scale
  int cut;                // bytes that come early (the lane in which the row ends loads the last 16)
};
// Vectors of up to 1024 take half a wave: its halves then hold rows of their own (FOLD 2), and a batch of four loads has eight rows,
// row 2 i + (lane / 32) in load i.
constexpr int kW4Short = 1024;

__device__ __forceinline__ W4Place w4_place(const W4Rows& w, int unit) {
  const int left = w.bytes - unit * (kW4Unit / 2);
  W4Place p = {0u, 0u, 0};  // (past the end: the row's first bytes, whose x is 0)
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
  for (int j = 0; j < kW4Unit / per; ++j) raw[j] = w4_bytes<16>(x + (unsigned)(min(unit * kW4Unit + j * per, k - per) * size));
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
      __builtin_amdgcn_sched_barrier(0);  // one after the other: together they take many registers
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
      w4_sums<XT>(raw[j], s, a);
      const w4_u4 p = w4_pairs(raw[j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) x.v[4 * j + e] = p[e];
    }
  }
  x.sum = s;
  plain |= !(a < kW4Large);
  return x;
}

// sum of (16 + q) x (16-bit x) or q x (FP32 x) over the lane's codes, for T vectors at once
template <int XT, int T>
__device__ __forceinline__ void w4_dot(w4_u4 codes, const W4X<XT> (&x)[T], float (&out)[T]) {
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
          a[t][0] = fmaf(q, __uint_as_float(x[t].v[8 * j + 2 * e]), a[t][0]);
          a[t][1] = fmaf(r, __uint_as_float(x[t].v[8 * j + 2 * e + 1]), a[t][1]);
        }
      }
    } else {
      unsigned b[4];
      w4_unpack<XT>(codes[j], b);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < T; ++t) {
          a[t][e % 2] = w4_dot2<XT>(b[e], x[t].v[4 * j + e], a[t][e % 2]);
        }
    }
  }
#pragma unroll
  for (int t = 0; t < T; ++t) out[t] = a[t][0] + a[t][1];
}

// A row of codes, its scales and its zero points.
struct W4Row {
  const uint8_t* codes;
  const char* scales;
  const uint8_t* zeros;
  int codes2, scales2, zeros2;  // FOLD 2: from the first half's row to the second's
  __device__ __forceinline__ W4Row of_half(bool second) const {
    if (!second) return *this;
    return {codes + codes2, scales + scales2, zeros + zeros2, 0, 0, 0};
  }
};
// Load `i` of a batch from row `first` on: row first + i (FOLD 1), or rows first + 2 i and the one behind (FOLD 2); rows past the end are
// the last.  The second of two rows is `other` rows behind.
template <int ST>
__device__ __forceinline__ W4Row w4_row(const W4Rows& w, int row) {
  const int64_t n = min(row, w.n - 1);
  return {w.codes + n * w.ld_codes, w.scales + n * w.ld_scales * (ST == OZ2_F32 ? 4 : 2), w.zeros + n * w.ld_zeros};
}
template <int ST, int FOLD>
__device__ __forceinline__ W4Row w4_row(const W4Rows& w, int first, int i) {
  W4Row r = w4_row<ST>(w, first + FOLD * i);
  r.codes2 = r.scales2 = r.zeros2 = 0;
  if (FOLD == 2 && first + 2 * i + 1 < w.n) r.codes2 = (int)w.ld_codes, r.scales2 = (int)w.ld_scales * (ST == OZ2_F32 ? 4 : 2), r.zeros2 = (int)w.ld_zeros;
  return r;
}

// The lane's sum of s (q - z) x straight from memory, one by one: for x with infinities, NaNs or values near the end of the range.
template <int XT, int ST, bool ZEROS>
__device__ __forceinline__ float w4_unit_plain(int k, int group, W4Row row, const char* x, int unit) {
  const int end = min((unit + 1) * kW4Unit, k), g = unit / (group / kW4Unit);
  float sum = 0.f;
#pragma unroll 1
  for (int i = unit * kW4Unit; i < end; ++i) {
    const int q = row.codes[i / 2] >> (i % 2 * 4) & 15;
    sum = fmaf(w4_load(ST, row.scales, g) * (float)(q - (ZEROS ? (int)row.zeros[g] : 8)), w4_load(XT, x, i), sum);
  }
  return sum;
}

// Sums of the four loads' values: of a batch's rows, lane 16 j (FOLD 1) holds row j; lanes 32 j and 32 j + 16 (FOLD 2) hold, in v[0] rows j and
// 2 + j, in v[1] rows 4 + j and 6 + j, and so do the 15 lanes behind each.
template <int FOLD>
__device__ __forceinline__ int w4_row_of_lane(int i) {
  const int lane = threadIdx.x % 64;
  return FOLD == 1 ? lane / 16 : 4 * i + lane / 32 + lane / 16 % 2 * 2;
}
template <int FOLD>
__device__ __forceinline__ void w4_sum4(float a, float b, float c, float d, float (&v)[FOLD]) {
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  auto swapped = [](u2 r) { return __uint_as_float(r[0]) + __uint_as_float(r[1]); };
  auto pair32 = [&](float p, float q) { return swapped(__builtin_amdgcn_permlane32_swap(__float_as_uint(p), __float_as_uint(q), false, false)); };
  auto pair16 = [&](float p, float q) { return swapped(__builtin_amdgcn_permlane16_swap(__float_as_uint(p), __float_as_uint(q), false, false)); };
  if constexpr (FOLD == 1) v[0] = pair16(pair32(a, c), pair32(b, d));
  else v[0] = pair16(a, b), v[1] = pair16(c, d);
#pragma unroll
  for (int i = 0; i < FOLD; ++i) v[i] += w4_partner<0>(v[i]), v[i] += w4_partner<1>(v[i]), v[i] += w4_partner<2>(v[i]), v[i] += w4_partner<3>(v[i]);
}

// Four loads of rows times T vectors, a span of the inner indexes; x as kept.  All loads come first: 4 KiB a wave in flight.
template <int XT, int T, int ST, bool ZEROS, int FOLD>
struct W4Rows4 {
  W4Regs<1, ST> r[4];

  template <class Row>
  __device__ __forceinline__ void fetch(Row row, W4Place at) {
    unsigned codes = at.codes, scale = at.group * (ST == OZ2_F32 ? 4 : 2), zero = at.group;
    asm volatile("" : "+v"(codes), "+v"(scale), "+v"(zero));  // (32 bits here: a loop would keep them widened, and add the row's address to that)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const W4Row p = row(i);
      const bool second = FOLD == 2 && threadIdx.x % 64 >= 32;
      r[i].q = w4_bytes<16>(p.codes + (codes + (unsigned)(second ? p.codes2 : 0)));
      r[i].s = w4_bytes<ST == OZ2_F32 ? 4 : 2>(p.scales + (scale + (unsigned)(second ? p.scales2 : 0)));
      if constexpr (ZEROS) r[i].z = p.zeros[zero + (unsigned)(second ? p.zeros2 : 0)];
    }
  }

  // sum[i][t] of the lane
  __device__ __forceinline__ void multiply(W4Place at, const W4X<XT> (&x)[T], bool ragged, float (&sum)[4][T]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w4_u4 q = r[i].q;
      if (ragged) q = w4_cut(q, at.cut);
      float s, z = 8.f, p[T];
      if constexpr (ST == OZ2_F32) s = __uint_as_float(r[i].s);
      else s = w4_decode16(ST, r[i].s);
      if constexpr (ZEROS) z = (float)r[i].z;
      w4_dot<XT, T>(q, x, p);
#pragma unroll
      for (int t = 0; t < T; ++t) sum[i][t] = s * fmaf(-(XT == OZ2_F32 ? z : z + kW4Offset), x[t].sum, p[t]);
    }
  }

  // The sums of the vectors in `which` again (no other's: what one vector holds changes no bit of another's result).
  template <class Row, class X>
  __device__ __forceinline__ void multiply_plain(unsigned which, int k, int group, Row row, X x, int unit, float (&sum)[4][T]) {
#pragma unroll 1
    for (int j = 0; j < 4 * T; ++j) {
      if (!(which >> (j % T) & 1)) continue;
      const float v = w4_unit_plain<XT, ST, ZEROS>(k, group, row(j / T).of_half(FOLD == 2 && threadIdx.x % 64 >= 32), x(j % T), unit);
      w4_each<4 * T>([&](auto i) __attribute__((always_inline)) {
        if (j == i.value) sum[i.value / T][i.value % T] = v;
      });
    }
  }
};

// T vectors of a span, from memory into registers; returns a bit for each vector whose values call for multiply_plain.  x(t): start of vector t.
template <int XT, int T, class X>
__device__ __forceinline__ unsigned w4_take_x(int k, int unit, X x, W4X<XT> (&kept)[T]) {
  w4_u4 raw[T][XT == OZ2_F32 ? 8 : 4];
  unsigned which = 0;
  asm volatile("" : "+v"(unit));  // else, in a loop, all that follows from it is kept in registers
#pragma unroll
  for (int t = 0; t < T; ++t) w4_load_x<XT>(x(t), k, unit, raw[t]);
#pragma unroll
  for (int t = 0; t < T; ++t) {
    bool plain = false;
    kept[t] = w4_keep_x<XT>(k, unit, raw[t], plain);
    which |= (unsigned)(__ballot(plain) != 0) << t;
  }
  return which;
}

#endif
#endif
