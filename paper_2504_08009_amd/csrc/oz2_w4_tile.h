// Two tiles of sixteen rows held in 4 bits times up to sixteen vectors, by one wave on the matrix cores.  Both tiles meet the same
// fragments of x, read from LDS once for the two.
//
// Four neighbouring lanes load 64 bytes of a row in one access; where each lane loads from a row of its own, as the matrix cores want their operand,
// the vector cache is asked 64 times for a load and sets the pace (65536 x 8192 with one vector: 3.6 TB/s).  The words then change lanes.
#ifndef OZ2_W4_TILE_H
#define OZ2_W4_TILE_H

#include "oz2_w4_core.h"

#ifdef __HIPCC__

constexpr int kW4Run = 4;  // blocks whose scales a wave loads together, a block a lane of four, and that it has in flight

// A tile as a launch sees it: its first row, and the lane's row (lane / 4) from there.
template <bool WIDE, bool ZEROS>
struct W4Tile {
  const uint8_t* codes;
  const char* scales;
  const uint8_t* zeros;
  unsigned codes_at, scales_at, zeros_at;

  __device__ __forceinline__ void init(const W4Rows& w, int row) {
    const int lane = threadIdx.x % 64, first = min(row, w.n - 1), mine = min(lane / 4, w.n - 1 - first);
    codes = w.codes + first * w.ld_codes, scales = w.scales + first * w.ld_scales * (WIDE ? 4 : 2), zeros = w.zeros + first * w.ld_zeros;
    codes_at = (unsigned)(mine * (int)w.ld_codes + lane % 4 * 16);
    scales_at = (unsigned)(mine * (int)w.ld_scales * (WIDE ? 4 : 2));
    zeros_at = (unsigned)(mine * (int)w.ld_zeros);
  }
};
inline bool w4_tile_fits(const W4Rows& w) {  // sixteen rows lie within 32 bits
  constexpr int64_t far = (int64_t)1 << 25;
  return w.ld_codes < far && w.ld_scales < far && w.ld_zeros < far;
}

template <int SPB, bool WIDE>
struct W4RunScales {
  typename W4Width<SPB * (WIDE ? 4 : 2)>::type s[2];
  typename W4Width<SPB>::type z[2];
};

// 32 bits that a loop must not keep widened, for the sake of loads with a scalar base
__device__ __forceinline__ unsigned w4_narrow(unsigned v) {
  asm volatile("" : "+v"(v));
  return v;
}

template <int XT, int SPB, int RT, bool WIDE, bool ZEROS>
struct W4Two {
  W4Tile<WIDE, ZEROS> tile[2];
  int half;  // whether 16-bit scales are f16
  int from, from_scale;  // lanes (times 4) whose codes, and whose scales of a run's first block, this lane takes

  __device__ __forceinline__ void init(int scale_type) {
    const int lane = threadIdx.x % 64;
    half = scale_type == OZ2_F16;
    from = (lane % 16 * 4 + lane / 16) * 4, from_scale = lane % 16 * 16;
  }
  __device__ __forceinline__ w4_u4 codes(int t, int block) const {
    return w4_bytes<16>(tile[t].codes + (int64_t)block * (kW4Block / 2) + w4_narrow(tile[t].codes_at));
  }
  __device__ __forceinline__ W4RunScales<SPB, WIDE> scales(const W4Rows& w, int run) const {
    constexpr int size = WIDE ? 4 : 2;
    W4RunScales<SPB, WIDE> r;
    const unsigned g = w4_group<SPB>(w, min(run * kW4Run + (int)(threadIdx.x % 4), w.full - 1));
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      r.s[t] = w4_bytes<SPB * size>(tile[t].scales + w4_narrow(tile[t].scales_at + g * size));
      if constexpr (ZEROS) r.z[t] = w4_bytes<SPB>(tile[t].zeros + w4_narrow(tile[t].zeros_at + g));
    }
    return r;
  }
  __device__ __forceinline__ float decode(unsigned v) const {
    const float b = __uint_as_float(v << 16), h = (float)__builtin_bit_cast(_Float16, (unsigned short)v);
    return half ? h : b;
  }

  // sum[t] += the tiles' products for one block.  q: codes as the matrix cores take them; scale(t, segment), zero(t, segment).
  template <class Scale, class Zero>
  __device__ __forceinline__ void block(const w4_u4 (&q)[2], Scale scale, Zero zero, const char* x, int part_bytes, float (&sum)[2][RT]) const {
    const int quarter = threadIdx.x % 64 / 16;
    constexpr unsigned one = XT == OZ2_F16 ? 0x3C003C00u : 0x3F803F80u;
    const unsigned ones[4] = {one, one, one, one};
    w4_each<SPB>([&](auto index) __attribute__((always_inline)) {
      constexpr int seg = index.value;
      w4_f4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}, of_x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4 / SPB; ++i) {
        const int j = seg * (4 / SPB) + i;
        unsigned b[2][4];
        w4_unpack<XT>(q[0][w4_register<SPB>(j)], b[0]);
        w4_unpack<XT>(q[1][w4_register<SPB>(j)], b[1]);
#pragma unroll
        for (int p = 0; p < w4_parts<XT>(); ++p) {
          const uint4 v = *reinterpret_cast<const uint4*>(x + p * part_bytes + 2 * w4_inner<SPB>(j, quarter));
          acc[0] = w4_mfma<XT>(v, b[0], acc[0]);
          acc[1] = w4_mfma<XT>(v, b[1], acc[1]);
          of_x = w4_mfma<XT>(v, ones, of_x);  // sum of x, as each lane wants it
        }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float s = scale(t, index), z = kW4Offset + zero(t, index);
#pragma unroll
        for (int i = 0; i < RT; ++i) sum[t][i] = fmaf(s, fmaf(-z, of_x[i], acc[t][i]), sum[t][i]);
      }
    });
  }

  // Loads of a first run, ahead of whatever has to be done before its products.  There is a whole block.
  struct Ahead {
    w4_u4 ring[kW4Run][2];
    W4RunScales<SPB, WIDE> now;
  };
  __device__ __forceinline__ void begin(const W4Rows& w, int first, int end, Ahead& a) const {
    a.now = scales(w, first);
    w4_each<kW4Run>([&](auto u) __attribute__((always_inline)) {
      const int b = max(min(first * kW4Run + u.value, end - 1), 0);
      a.ring[u.value][0] = codes(0, b), a.ring[u.value][1] = codes(1, b);
    });
  }
  // Runs first, first + stride, ... (`count` of them) of the whole blocks below `end`.  x: of block `origin`.
  __device__ __forceinline__ void multiply(const W4Rows& w, int first, int stride, int count, int end, int origin, Ahead& ahead, const char* x, int part_bytes,
                                           float (&sum)[2][RT]) const {
    w4_u4 (&ring)[kW4Run][2] = ahead.ring;
    W4RunScales<SPB, WIDE> now = ahead.now, next;
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
      const int run = first + i * stride, then = i + 1 < count ? run + stride : run;
      next = scales(w, then);
      w4_each<kW4Run>([&](auto u) __attribute__((always_inline)) {
        const int b = run * kW4Run + u.value;
        if (b < end) {
          w4_u4 q[2];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int j = 0; j < 4; ++j) q[t][j] = __builtin_amdgcn_ds_bpermute(from, ring[u.value][t][j]);
            q[t] = w4_exchange<SPB>(q[t]);
          }
          constexpr int words = (SPB * (WIDE ? 4 : 2) + 3) / 4;
          unsigned s[2][words], z[2];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int j = 0; j < words; ++j)
              s[t][j] = __builtin_amdgcn_ds_bpermute(from_scale + 4 * u.value, w4_word<SPB * (WIDE ? 4 : 2)>(now.s[t], j));
            if constexpr (ZEROS) z[t] = __builtin_amdgcn_ds_bpermute(from_scale + 4 * u.value, w4_word<SPB>(now.z[t], 0));
          }
          block(
              q,
              [&](int t, auto seg) __attribute__((always_inline)) {
                if constexpr (WIDE) return __uint_as_float(s[t][seg.value]);
                else return decode(s[t][seg.value / 2] >> (seg.value % 2 * 16));
              },
              [&](int t, auto seg) __attribute__((always_inline)) {
                if constexpr (ZEROS) return (float)(z[t] >> (8 * seg.value) & 255u);
                else return 8.f;
              },
              x + (b - origin) * kW4Block * 2, part_bytes, sum);
        }
        const int f = min(then * kW4Run + u.value, end - 1);
        ring[u.value][0] = codes(0, f), ring[u.value][1] = codes(1, f);
      });
      now = next;
    }
  }

  // The block behind the whole ones; row[t]: the tiles' first rows.
  __device__ __forceinline__ void multiply_tail(const W4Rows (&w)[2], const int (&row)[2], const char* x, int part_bytes, float (&sum)[2][RT]) const {
    constexpr int ST = WIDE ? OZ2_F32 : OZ2_BF16;  // (16 bits are decoded here)
    W4Tail<SPB> r[2];
    w4_u4 q[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) r[t] = w4_fetch_tail<SPB, ST, ZEROS>(w[t], w4_lane<ST>(w[t], row[t] + threadIdx.x % 16));
#pragma unroll
    for (int t = 0; t < 2; ++t) q[t] = w4_exchange<SPB>(w4_cut(r[t].q, r[t].cut));
    const int g = w4_group<SPB>(w[0], w[0].full);
    block(
        q,
        [&](int t, auto i) __attribute__((always_inline)) {  // (0 past the last group: a scale that is not finite must not meet the 0 of x)
          const float s = WIDE ? __uint_as_float(r[t].s[i.value]) : decode(r[t].s[i.value]);
          return g + i.value < w[0].groups ? s : 0.f;
        },
        [&](int t, auto i) __attribute__((always_inline)) { return (float)r[t].z[i.value]; }, x, part_bytes, sum);
  }

  // The sums over block b by the formula itself: for x with infinities, NaNs or values near the end of the range, from which the
  // products above make sums that are not finite, and only from these.  value(r, k): x of the lane's token quarter + 4 r.
  template <class X>
  __device__ __forceinline__ void block_plain(const W4Rows (&w)[2], const int (&row)[2], int b, X value, float (&sum)[2][RT]) const {
    const int end = min(w[0].k, (b + 1) * kW4Block);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const W4Lane l = w4_lane<WIDE ? OZ2_F32 : OZ2_BF16>(w[t], row[t] + threadIdx.x % 16);
      const uint8_t* code = l.codes - threadIdx.x % 64 / 16 * 16;
#pragma unroll 1
      for (int i = b * kW4Block; i < end; ++i) {
        const int g = SPB > 1 ? i / (kW4Block / SPB) : w4_group<1>(w[t], b);
        const float s = WIDE ? reinterpret_cast<const float*>(l.scales)[g] : decode(reinterpret_cast<const uint16_t*>(l.scales)[g]);
        const float v = s * (float)((code[i / 2] >> (i % 2 * 4) & 15) - (ZEROS ? (int)l.zeros[g] : 8));
#pragma unroll
        for (int r = 0; r < RT; ++r) sum[t][r] = fmaf(v, value(r, i), sum[t][r]);
      }
    }
  }
};

// Brings blocks start .. start + length - 1 of x into LDS, zeros past k, by all threads of a workgroup, between two barriers of the caller's.  A thread
// takes eight values of several tokens at a time.  row(token): element offset of the vector; k is at least 8.
template <int XT, class Row>
__device__ __forceinline__ void w4_stage(const char* x, Row row, int tokens, int k, int start, int length, char* lds, int pitch, int threads) {
  constexpr int PIECES = XT == OZ2_F32 ? 4 : 8, P = w4_parts<XT>(), size = XT == OZ2_F32 ? 4 : 2, per = 16 / size;  // 128 bytes of a thread in flight
#pragma unroll 1
  for (int e = threadIdx.x; e < length * (kW4Block / 8); e += threads) {
    const int at = start * kW4Block + e * 8;
#pragma unroll 1
    for (int t = 0; t < tokens; t += PIECES) {
      w4_u4 raw[PIECES][8 / per];
      w4_each<PIECES>([&](auto i) __attribute__((always_inline)) {
        const char* p = x + row(min(t + i.value, tokens - 1)) * size;
        w4_each<8 / per>([&](auto h) __attribute__((always_inline)) { raw[i.value][h.value] = w4_bytes<16>(p + w4_narrow(min(at + h.value * per, k - per) * size)); });
      });
      if (at + 8 > k)  // the 16 bytes that end with the vector, or nothing
        w4_each<PIECES>([&](auto i) __attribute__((always_inline)) {
          w4_each<8 / per>([&](auto h) __attribute__((always_inline)) {
            const int there = k - (at + h.value * per);
            w4_u4& v = raw[i.value][h.value];
            v = there <= 0 ? w4_u4{0, 0, 0, 0} : there < per ? w4_cut(v, (per - there) * size) : v;
          });
        });
      w4_each<PIECES>([&](auto i) __attribute__((always_inline)) {
        if (t + i.value >= tokens) return;
        char* to = lds + (t + i.value) * P * pitch + 16 * e;
        if constexpr (XT == OZ2_F32) {
          unsigned h[P][8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {  // cut, not rounded: each part takes the next eight bits, and none can overflow
            float rest = __uint_as_float(raw[i.value][j / 4][j % 4]);
#pragma unroll
            for (int c = 0; c < P; ++c) {
              h[c][j] = __float_as_uint(rest);
              rest -= __uint_as_float(h[c][j] & 0xFFFF0000u);
            }
          }
#pragma unroll
          for (int c = 0; c < P; ++c)
            *reinterpret_cast<w4_u4*>(to + c * pitch) =
                w4_u4{__builtin_amdgcn_perm(h[c][4], h[c][0], 0x07060302u), __builtin_amdgcn_perm(h[c][5], h[c][1], 0x07060302u),
                      __builtin_amdgcn_perm(h[c][6], h[c][2], 0x07060302u), __builtin_amdgcn_perm(h[c][7], h[c][3], 0x07060302u)};
        } else {
          *reinterpret_cast<w4_u4*>(to) = w4_pairs(raw[i.value][0]);
        }
      });
    }
  }
}

#endif
#endif
