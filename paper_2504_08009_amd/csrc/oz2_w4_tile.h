// Two tiles of sixteen rows held in 4 bits times up to sixteen vectors, by one wave on the matrix cores.  Both tiles meet the same
// fragments of x, read from LDS once for the two.  Sums of (q - z) x come from those of (16 + q) x and of x, the latter formed by the matrix cores
// as well, with an operand of equal values.
//
// Bound, at the sizes measured, by what comes before and after a wave's few blocks (x into LDS, the first loads' way, sums over the waves)
// and by the instructions that turn codes into operands, not by bytes: 8192 x 8192 with 16 vectors takes 18.7 us for 35 MB (1.9 TB/s), the
// experts of 32 tokens, 8 of 128 of 4096 x 2048, 437 us for 1.58 GB (3.6 TB/s).
//
// Four neighbouring lanes load 64 bytes of a row, eight of them two lines' worth of two blocks; where each lane loads from a row of its own, as the matrix
// cores want their operand, the vector cache is asked 64 times for a load and sets the pace.  The words then change lanes and
// registers: inside four lanes by selecting from the neighbour's, across sixteen and 32 by swapping registers' halves, so that LDS
// is left to x.
#ifndef OZ2_W4_TILE_H
#define OZ2_W4_TILE_H

#include "oz2_w4_core.h"

#ifdef __HIPCC__

constexpr int kW4Run = 2;   // blocks that a wave loads together
constexpr int kW4Ahead = 2; // runs in flight

inline bool w4_tile_fits(const W4Rows& w) {  // a lane's rows lie within 32 bits of each other
  constexpr int64_t far = (int64_t)1 << 25;
  return w.ld_codes < far && w.ld_scales < far && w.ld_zeros < far;
}

// 32 bits that a loop must not keep widened, for the sake of loads with a scalar base
__device__ __forceinline__ unsigned w4_narrow(unsigned v) {
  asm volatile("" : "+v"(v));
  return v;
}

template <int XT, int SPB, int RT, bool WIDE, bool ZEROS>
struct W4Two {
  // Where a lane loads from.  Codes: load j takes row 4 (lane / 4 % 4) + j of tile lane / 16 % 2, chunk lane % 4 of block lane / 32 of the run;
  // scales: row lane % 16 of that tile and block.
  const uint8_t* codes;
  const char* scales;
  const uint8_t* zeros;
  int step[3];  // from the lane's first row to the others (fewer at the end of the matrix: the last one again)
  int half;     // whether 16-bit scales are f16

  __device__ __forceinline__ void init(const W4Rows (&w)[2], const int (&row)[2], int scale_type) {
    const int lane = w4_thread() % 64, t = lane / 16 % 2;
    half = scale_type == OZ2_F16;
    const W4Rows& m = w[0];  // (both are alike but for their addresses)
    const int n = m.n - 1, first = min((t ? row[1] : row[0]) + lane / 4 % 4 * 4, n), mine = min((t ? row[1] : row[0]) + lane % 16, n);
    codes = (t ? w[1].codes : w[0].codes) + first * (t ? w[1].ld_codes : w[0].ld_codes) + lane % 4 * 16;
    scales = (t ? w[1].scales : w[0].scales) + mine * (t ? w[1].ld_scales : w[0].ld_scales) * (WIDE ? 4 : 2);
    zeros = (t ? w[1].zeros : w[0].zeros) + mine * (t ? w[1].ld_zeros : w[0].ld_zeros);
#pragma unroll
    for (int j = 0; j < 3; ++j) step[j] = min(j + 1, n - first) * (int)(t ? w[1].ld_codes : w[0].ld_codes);
  }
  struct Run {
    w4_u4 q[4];
    typename W4Width<SPB * (WIDE ? 4 : 2)>::type s;
    typename W4Width<SPB>::type z;
  };
  // The run's blocks below `end`; of those past it, the one before it.
  __device__ __forceinline__ Run fetch(const W4Rows& w, int run, int end) const {
    constexpr int size = WIDE ? 4 : 2;
    Run r;
    const int b = min(run * kW4Run + (int)(threadIdx.x % 64 / 32), end - 1);
    const unsigned at = b * (kW4Block / 2), g = w4_group<SPB>(w, b);
#pragma unroll
    for (int j = 0; j < 4; ++j) r.q[j] = w4_bytes<16>(codes + (unsigned)(at + (j ? step[j ? j - 1 : 0] : 0)));
    r.s = w4_bytes<SPB * size>(scales + g * size);
    if constexpr (ZEROS) r.z = w4_bytes<SPB>(zeros + g);
    return r;
  }
  __device__ __forceinline__ float decode(unsigned v) const {
    const float b = __uint_as_float(v << 16), h = (float)__builtin_bit_cast(_Float16, (unsigned short)v);
    return half ? h : b;
  }
  // Register j of lane i for register i of lane j, of every four lanes: two exchanges, of which each result is one instruction, the lane's own
  // value or its neighbour's by a mask.  The waits are those between a vector instruction and one that reads its result from another lane: before
  // the first, for what the compiler puts ahead, and behind the last, for what it puts there (it counts nothing in here as such a writer).
  static __device__ __forceinline__ void turn_four(unsigned& a, unsigned& b, unsigned& c, unsigned& d) {
    unsigned p, q, r, s;
    asm("s_nop 1\n\t"
        "s_mov_b64 vcc, %8\n\t"
        "v_cndmask_b32_dpp %1, %4, %5, vcc quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
        "v_cndmask_b32_dpp %3, %6, %7, vcc quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
        "s_not_b64 vcc, vcc\n\t"
        "v_cndmask_b32_dpp %0, %5, %4, vcc quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
        "v_cndmask_b32_dpp %2, %7, %6, vcc quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
        "s_mov_b64 vcc, %9\n\t"
        "v_cndmask_b32_dpp %6, %0, %2, vcc quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
        "v_cndmask_b32_dpp %7, %1, %3, vcc quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
        "s_not_b64 vcc, vcc\n\t"
        "v_cndmask_b32_dpp %4, %2, %0, vcc quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
        "v_cndmask_b32_dpp %5, %3, %1, vcc quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
        "s_nop 1\n\t"
        : "=&v"(p), "=&v"(q), "=&v"(r), "=&v"(s), "+v"(a), "+v"(b), "+v"(c), "+v"(d)
        : "s"(0xAAAAAAAAAAAAAAAAull), "s"(0xCCCCCCCCCCCCCCCCull)
        : "vcc", "scc");
  }
  // out[2 block + tile]: codes as the matrix cores take them
  static __device__ __forceinline__ void turn(const Run& r, w4_u4 (&out)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      unsigned v[4] = {r.q[0][j], r.q[1][j], r.q[2][j], r.q[3][j]};
      turn_four(v[0], v[1], v[2], v[3]);
      const w4_u4 u = w4_exchange<4>(w4_u4{v[0], v[1], v[2], v[3]});
#pragma unroll
      for (int i = 0; i < 4; ++i) out[i][j] = u[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = w4_exchange<SPB>(out[i]);
  }
  // out[2 block + tile]: the value of the lane's row
  static __device__ __forceinline__ void spread(float f, float (&out)[4]) {
    const unsigned v = __float_as_uint(f);
    typedef unsigned u2 __attribute__((ext_vector_type(2)));
    const u2 r = __builtin_amdgcn_permlane16_swap(v, v, false, false);  // tile 0's, tile 1's in the sixteens of either block's 32
    const u2 a = __builtin_amdgcn_permlane32_swap(r[0], r[0], false, false), b = __builtin_amdgcn_permlane32_swap(r[1], r[1], false, false);
    out[0] = __uint_as_float(a[0]), out[1] = __uint_as_float(b[0]), out[2] = __uint_as_float(a[1]), out[3] = __uint_as_float(b[1]);
  }

  // sum[t] += the tiles' products for one block.  q: codes as the matrix cores take them; scale(t, segment), zero(t, segment).
  template <class Scale, class Zero>
  __device__ __forceinline__ void block(const w4_u4 (&q)[2], Scale scale, Zero zero, const char* x, int part_bytes, float (&sum)[2][RT]) const {
    const int quarter = threadIdx.x % 64 / 16;
    // sum (16 + q) x - 24 sum x comes out of the matrix cores where there are no zero points, else sum (16 + q) x and sum x
    constexpr unsigned one = ZEROS ? (XT == OZ2_F16 ? 0x3C003C00u : 0x3F803F80u) : (XT == OZ2_F16 ? 0xCE00CE00u : 0xC1C0C1C0u);
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
          of_x = w4_mfma<XT>(v, ones, of_x);
          acc[0] = w4_mfma<XT>(v, b[0], acc[0]);
          acc[1] = w4_mfma<XT>(v, b[1], acc[1]);
        }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float s = scale(t, index);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          const float v = ZEROS ? fmaf(-(kW4Offset + zero(t, index)), of_x[i], acc[t][i]) : acc[t][i] + of_x[i];
          sum[t][i] = fmaf(s, v, sum[t][i]);
        }
      }
    });
  }

  // What a wave walks: runs first, first + stride, ... (`count` of them) of the whole blocks below `end`, from the `turn`-th on and round.  Each wave
  // begins at a place of its own: rows lie whole pages apart as a rule, and where all stand at the same inner index, they ask the same few memory channels.
  struct Walk {
    int first, stride, count, end, turn;
    __device__ __forceinline__ Walk(int first, int stride, int count, int end, unsigned who)
        : first(first), stride(stride), count(count), end(end), turn(count > 1 ? who % (unsigned)count : 0) {}
    __device__ __forceinline__ int run(int i) const {  // (past the last: the last again)
      i = max(min(i, count - 1), 0) + turn;
      return first + (i < count || count < 1 ? i : i - count) * stride;
    }
  };
  // Loads of the first runs, ahead of whatever has to be done before their products.
  struct Ahead {
    Run run[kW4Ahead];
  };
  __device__ __forceinline__ void begin(const W4Rows& w, const Walk& walk, Ahead& a) const {
    w4_each<kW4Ahead>([&](auto i) __attribute__((always_inline)) { a.run[i.value] = fetch(w, walk.run(i.value), max(walk.end, 1)); });
  }
  // x: of block `origin`.
  __device__ __forceinline__ void multiply(const W4Rows& w, const Walk& walk, int origin, Ahead& ahead, const char* x, int part_bytes, float (&sum)[2][RT]) const {
#pragma unroll 1
    for (int i = 0; i < walk.count; i += kW4Ahead)
      w4_each<kW4Ahead>([&](auto a) __attribute__((always_inline)) {
        const int at = i + a.value, run = walk.run(at);
        w4_u4 q[4];
        float s[SPB][4], z[SPB][4];
        turn(ahead.run[a.value], q);
        w4_each<SPB>([&](auto j) __attribute__((always_inline)) {  // (decoded where they were loaded, once, and not where they are used)
          const auto& r = ahead.run[a.value];
          if constexpr (WIDE) spread(__uint_as_float(w4_word<SPB * 4>(r.s, j.value)), s[j.value]);
          else spread(decode(w4_word<SPB * 2>(r.s, j.value / 2) >> (j.value % 2 * 16)), s[j.value]);
          if constexpr (ZEROS) spread((float)(w4_word<SPB>(r.z, 0) >> (8 * j.value) & 255u), z[j.value]);
        });
        ahead.run[a.value] = fetch(w, walk.run(at + kW4Ahead), walk.end);
        w4_each<kW4Run>([&](auto u) __attribute__((always_inline)) {
          const int b = run * kW4Run + u.value;
          if (at < walk.count && b < walk.end) {
            const w4_u4 codes_of[2] = {q[2 * u.value], q[2 * u.value + 1]};
            block(
                codes_of, [&](int t, auto seg) __attribute__((always_inline)) { return s[seg.value][2 * u.value + t]; },
                [&](int t, auto seg) __attribute__((always_inline)) { return z[seg.value][2 * u.value + t]; },
                x + (b - origin) * kW4Block * 2, part_bytes, sum);
          }
        });
      });
  }

  // The block behind the whole ones; row[t]: the tiles' first rows.
  __device__ __forceinline__ void multiply_tail(const W4Rows (&w)[2], const int (&row)[2], const char* x, int part_bytes, float (&sum)[2][RT]) const {
    constexpr int ST = WIDE ? OZ2_F32 : OZ2_BF16;  // (16 bits are decoded here)
    W4Tail<SPB> r[2];
    w4_u4 q[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) r[t] = w4_fetch_tail<SPB, ST, ZEROS>(w[t], w4_lane<ST>(w[t], row[t] + w4_thread() % 16));
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
      const W4Lane l = w4_lane<WIDE ? OZ2_F32 : OZ2_BF16>(w[t], row[t] + w4_thread() % 16);
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
// takes eight values of several tokens at a time.  vector(token): its start; k is at least 8.
template <int XT, class X>
__device__ __forceinline__ void w4_stage(X vector, int tokens, int k, int start, int length, char* lds, int pitch, int threads) {
  constexpr int PIECES = XT == OZ2_F32 ? 4 : 8, P = w4_parts<XT>(), size = XT == OZ2_F32 ? 4 : 2, per = 16 / size;  // 128 bytes of a thread in flight
#pragma unroll 1
  for (int e = w4_thread(); e < length * (kW4Block / 8); e += threads) {
    const int at = start * kW4Block + e * 8;
#pragma unroll 1
    for (int t = 0; t < tokens; t += PIECES) {
      w4_u4 raw[PIECES][8 / per];
      w4_each<PIECES>([&](auto i) __attribute__((always_inline)) {
        const char* p = vector(min(t + i.value, tokens - 1));
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
