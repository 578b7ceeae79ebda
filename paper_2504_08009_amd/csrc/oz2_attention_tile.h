// Attention over packed prompts in BF16 and FP16 on the matrix cores: the kernel of one type and of dims up to DP.
//
// A workgroup has 256, 128 or 64 rows, a wave 32 of them, which are the columns of its products (32 x 32 x 16): keys x rows, then dims x rows.  So a lane has one
// row throughout, maxima and sums stay in lanes, and what it holds of the first product, rounded, is its part of the second one's operand as it is: of sixteen
// keys the lanes' lower half has 0..3 and 8..11, the upper half 4..7 and 12..15, and the values are read in that order.  (p is rounded to the type of the values,
// as the matrix cores take it; its sum l is of what it was before.  In FP16 that is half a step, 2^-11 of p, or 2^-32 of the largest p where that is more.)
//   Keys and values come into LDS in tiles of 64, in two buffers, by copies that pass no registers, begun a tile ahead; one barrier a tile.  Values are wanted with
// keys along a lane's words: ds_read_b64_tr_b16 turns 4 x 16 of them on their way.
//   A step takes 32 keys, and works on three of them at once, none of which waits for another: scores of step j + 1 and values of step j - 1 on the matrix cores, the
// exponentials of step j on the vector units.  m follows the maximum only where a score is more than 8 above it (to base 2), which hardly happens after the
// first tile; so the sums are hardly ever rescaled.  `step` is for tiles that all rows see, and has no branch but that; `last_step` is for all others.
//   With SPLIT = 2 the two halves of a workgroup have the same rows and every other tile of keys each; their sums are joined at the end.
//   16384 tokens of 16 heads of 128 values, FP16, causal, take 1.03 to 1.10 ms, 1000 to 1070 TFLOP/s, where a large matrix product reaches 1507: the vector units' part of
// a step, sixteen exponentials a lane and what goes with them, is nearly as long as the products' 16 x 32 cycles, and the clock falls under both.
#ifndef OZ2_ATTENTION_TILE_H
#define OZ2_ATTENTION_TILE_H

#include "oz2_attention.h"
#include "oz2_gemm.h"
#include "oz2_w4_core.h"

#ifdef __HIPCC__

typedef float at_f16 __attribute__((ext_vector_type(16)));
typedef short at_s4 __attribute__((ext_vector_type(4)));
typedef unsigned at_u2 __attribute__((ext_vector_type(2)));

constexpr int kTileKeys = 64;

template <int XT>
__device__ __forceinline__ at_f16 at_mfma(w4_u4 a, w4_u4 b, at_f16 c) {
  if constexpr (XT == OZ2_F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(w4_h8, a), __builtin_bit_cast(w4_h8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(w4_bf8, a), __builtin_bit_cast(w4_bf8, b), c, 0, 0, 0);
}
template <int XT>
__device__ __forceinline__ unsigned at_pair(float a, float b) {
  typedef float Two __attribute__((ext_vector_type(2)));
  typedef _Float16 Half __attribute__((ext_vector_type(2)));
  typedef __bf16 Brain __attribute__((ext_vector_type(2)));
  if constexpr (XT == OZ2_F16) return __builtin_bit_cast(unsigned, __builtin_convertvector((Two{a, b}), Half));
  else return __builtin_bit_cast(unsigned, __builtin_convertvector((Two{a, b}), Brain));
}
template <int XT>
__device__ __forceinline__ float at_value(unsigned w, int upper) {
  if constexpr (XT == OZ2_F16) return (float)__builtin_bit_cast(_Float16, (uint16_t)(upper ? w >> 16 : w));
  else return __uint_as_float(upper ? w & 0xffff0000u : w << 16);
}
// whether either of a pair is not finite
template <int XT>
__device__ __forceinline__ bool at_odd(unsigned w) {
  constexpr unsigned top = XT == OZ2_F16 ? 0x7c00u : 0x7f80u;
  return (w & top) == top || (w & top << 16) == top << 16;
}

// load_to_lds_16 for the lanes of `lanes` alone; what others would have written is left as it was.
__device__ __forceinline__ void at_load_of(const int8_t* base, unsigned voff, unsigned lds_addr, unsigned long long lanes) {
  unsigned long long all;
  asm volatile(
      "s_mov_b32 m0, %3\n\t"
      "s_and_saveexec_b64 %0, %4\n\t"
      "global_load_lds_dwordx4 %1, %2\n\t"
      "s_mov_b64 exec, %0"
      : "=&s"(all)
      : "v"(voff), "s"(base), "s"(lds_addr), "s"(lanes)
      : "memory", "m0", "scc");
}

template <int XT, int DP, int WAVES, int SPLIT>
__global__ void __launch_bounds__(64 * WAVES, DP <= 64 ? 3 : DP <= 128 ? 2 : 1) attention_tile_kernel(Attention a) {
  constexpr int E = DP / 16, F = DP / 32, ROW = DP <= 64 ? 128 : DP <= 128 ? 256 : 512;  // bytes of a row in LDS
  constexpr int THREADS = 64 * WAVES / SPLIT, ROWS = 32 * WAVES / SPLIT, TILE = kTileKeys * ROW;
  constexpr int LOADS = TILE / 16 / THREADS, LDS = 4 * TILE;  // keys, keys, values, values
  // m is the maximum less UP: in FP16, where normal numbers end at 2^-14, p goes up to 2^15, and many keys far below one count
  constexpr float UP = XT == OZ2_F16 ? 7.f : 0.f;
  __shared__ __attribute__((aligned(16))) char all_lds[SPLIT * LDS];  // of each part
  __shared__ int all_odd[SPLIT][2];                            // whether the tile of values has one that is not finite, of even and odd tiles
  __shared__ unsigned weights[WAVES][8][32];              // (where it has: p of two keys)

  const int tiles = (int)((unsigned)gridDim.x / (unsigned)a.kv_heads);
  const int head = blockIdx.x % a.kv_heads, lane = threadIdx.x % 64, col = lane % 32, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), part = wave / (WAVES / SPLIT), thread = threadIdx.x % THREADS;
  char* const lds = all_lds + part * LDS;
  int* const odd = all_odd[part];
  if (thread < 2) odd[thread] = 0;
  const AttentionTile tile = attention_tile(a, blockIdx.x / a.kv_heads, tiles, ROWS);
  const int rows = tile.tokens * a.group;
  if (tile.first >= rows) return;

  // The part's keys: every SPLIT-th tile, counted as if they were one behind the other.  `own` of the first n keys belong to it.
  auto own = [&](int n) {
    if constexpr (SPLIT == 1) return n;
    const int full = n / kTileKeys, mine = full > part ? (full - part + SPLIT - 1) / SPLIT : 0;
    return mine * kTileKeys + (full % SPLIT == part ? n % kTileKeys : 0);
  };
  // keys that the wave's rows see at all, and that all of them see; and the most of any part
  const int first_row = tile.first + wave % (WAVES / SPLIT) * 32, last_row = min(first_row + 32, rows) - 1;
  const int end = first_row >= rows ? 0 : own(a.causal ? last_row / a.per_group + 1 : tile.tokens);
  const int full = first_row >= rows ? 0 : own(a.causal ? first_row / a.per_group + 1 : tile.tokens);
  const int seen_by_any = a.causal ? min(tile.first + ROWS - 1, rows - 1) / a.per_group + 1 : tile.tokens, tokens = own(tile.tokens);
  const int all = own(seen_by_any), most = SPLIT == 1 ? all : min(seen_by_any, (seen_by_any / (SPLIT * kTileKeys) + 1) * kTileKeys);
  const int steps = (end + 31) / 32, groups = (((most + 31) / 32) + 1) / 2;
  // groups whose steps, and the next one, all rows of the workgroup see: of the last part, which has the fewest keys
  const int seen_by_all = a.causal ? tile.first / a.per_group + 1 : tile.tokens;
  const int least = SPLIT == 1 ? seen_by_all : seen_by_all / (SPLIT * kTileKeys) * kTileKeys;
  const int easy = least >= 96 ? (least - 96) / 64 + 1 : 0;

  w4_u4 q[E];
  const int row = min(first_row + col, rows - 1), at = row / a.per_group;
  const int64_t query = (int64_t)head * a.group + (row - at * a.group);
  const int sees = own(a.causal ? at + 1 : tile.tokens);
  const uint16_t* from = static_cast<const uint16_t*>(a.q.data) + (tile.begin + at) * a.q.ld_token + query * a.q.ld_head;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int d = 16 * e + 8 * half;
    q[e] = w4_u4{0, 0, 0, 0};
    if (d < a.dim) q[e] = *reinterpret_cast<const w4_u4*>(from + d);
  }

  // Copies of tiles into LDS: sixteen bytes a lane, a wave's 1024 beside each other.  Pieces of sixteen bytes change places within a row, so that sixteen keys' pieces, and
  // four values' 64 bytes, lie in all banks: which piece comes to a place is chosen by what the lane loads.  Rows behind the last token are copies of it, which no row
  // sees.  Pieces behind the last dim: of keys 0 from the beginning on, and not copied to (they meet a 0 of q, which an infinity would make a NaN); of values the first
  // piece, whose sums are not stored.
  constexpr int PIECES = ROW / 16, PER = THREADS / PIECES, TURNS = PER % 16 ? 2 : 1;
  const int of_key = thread / PIECES, place = thread % PIECES;
  static_assert(TURNS == 1 || PER % 16 == 8, "a thread's keys have one exchange of pieces, or two in turn");
  const int k_piece = place ^ (ROW == 128 ? of_key / 2 % 8 : of_key % 16);  // (of odd loads with two turns: k_piece ^ 8)
  unsigned long long k_lanes[TURNS];
#pragma unroll
  for (int t = 0; t < TURNS; ++t) k_lanes[t] = __ballot((k_piece ^ t * 8) * 8 < a.dim);
  const int v_swizzled = place ^ (ROW == 128 ? of_key / 2 % 2 : of_key % 4) * 4;
  unsigned pieces = k_piece * 16 | (v_swizzled * 8 < a.dim ? v_swizzled : 0) << 20;  // (bytes of both in one register, which is short of others' in the loops)
  const char* k_from = static_cast<const char*>(a.k.data) + (tile.begin * a.k.ld_token + head * a.k.ld_head) * 2;
  const char* v_from = static_cast<const char*>(a.v.data) + (tile.begin * a.v.ld_token + head * a.v.ld_head) * 2;
  const int k_step = (int)(a.k.ld_token * 2), v_step = (int)(a.v.ld_token * 2);
  const unsigned lds_at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds + wave % (WAVES / SPLIT) * 1024;
  auto fetch = [&](const char* from, int step, int first, auto load) {  // (steps below 2^24)
    const int last = min(kTileKeys, tokens - first) - 1;
    int key = of_key;
    if constexpr (DP <= 128) asm volatile("" : "+v"(key), "+v"(pieces));  // (else what follows from them is held in registers across the loops)
    from += (int64_t)(SPLIT > 1 ? first * SPLIT + part * kTileKeys : first) * step;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int at = min(key + i * PER, last);
      // (of more dims a piece of q was spilled in FP16 with the one product or the other line, which every step then waited for: 4096 tokens of 16 heads of 256 213 us, 190 so)
      load(reinterpret_cast<const int8_t*>(from), DP <= 128 ? __umul24(at, step) : (unsigned)(at * step), i);
    }
  };
  auto fetch_keys = [&](int number) {
    fetch(k_from, k_step, number * kTileKeys, [&](const int8_t* from, unsigned at, int i) {
      at_load_of(from, at + ((pieces & 0xffff) ^ i % TURNS * 128), lds_at + number % 2 * TILE + i * THREADS * 16, k_lanes[i % TURNS]);
    });
  };
  auto fetch_values = [&](int number) {
    fetch(v_from, v_step, number * kTileKeys, [&](const int8_t* from, unsigned at, int i) {
      load_to_lds_16(from, at + (pieces >> 16), lds_at + (2 + number % 2) * TILE + i * THREADS * 16);
    });
  };
#pragma unroll
  for (int t = 0; t < TURNS; ++t)
    if ((k_piece ^ t * 8) * 8 >= a.dim)
#pragma unroll
      for (int i = t; i < 2 * LOADS; i += TURNS) *reinterpret_cast<w4_u4*>(lds + (i * THREADS + thread) * 16) = w4_u4{0, 0, 0, 0};
  static_assert(LOADS % TURNS == 0, "both tiles of keys have the same turns");

  // where a lane reads: pieces of keys and 64 bytes of values at these with bits exchanged
  const int k_at = col * ROW + (half ^ (ROW == 128 ? col / 2 % 8 : col % 16)) * 16;
  const int v_at = 2 * TILE + (4 * half + lane % 16 / 4) * ROW + (ROW == 128 ? lane % 16 / 8 : lane % 16 / 4) * 64 + lane / 16 % 2 * 32 + lane % 4 * 8;

  float m = kNoScore, l = 0.f, scale2 = a.scale2;
  at_f16 o[F], s[2];
  w4_u4 p[2][2];
#pragma unroll
  for (int f = 0; f < F; ++f)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[f][i] = 0.f;

  // (at: bytes from the first tile of keys, or of values)
  auto key_piece = [&](int at, int e) { return *reinterpret_cast<const w4_u4*>(lds + ((at + k_at) ^ (e * 32))); };
  auto value_piece = [&](int at, int b, int f) {
    typedef __attribute__((address_space(3))) at_s4* In;
    const char* from = lds + ((at + v_at) ^ (f * 64));
    const at_s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((In)(from + 16 * b * ROW));
    const at_s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((In)(from + (16 * b + 8) * ROW));
    const at_u2 l2 = __builtin_bit_cast(at_u2, lo), h2 = __builtin_bit_cast(at_u2, hi);
    return w4_u4{l2[0], l2[1], h2[0], h2[1]};
  };
  auto clear_scores = [&](at_f16 &s) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
  };
  auto score_with = [&](at_f16 &s, int at, int e) {
    const w4_u4 k = key_piece(at, e);
    s = at_mfma<XT>(k, q[e], s);
  };
  auto add_with = [&](const w4_u4 (&p)[2], int at, int b, int f) {
    const w4_u4 v = value_piece(at, b, f);
    o[f] = at_mfma<XT>(v, p[b], o[f]);
  };
  auto score = [&](at_f16 &s, int at) {
    clear_scores(s);
#pragma unroll
    for (int e = 0; e < E; ++e) score_with(s, at, e);
  };
  auto add = [&](const w4_u4 (&p)[2], int at) {
#pragma unroll
    for (int i = 0; i < 2 * F; ++i) add_with(p, at, i / F, i % F);
  };
  // what lanes of a wave have written is there for its others, and what they have read may be written over
  auto exchanged = [&]() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  };
  // The same with values that are not finite, for rows that do not see all of them: key by key.
  auto add_seen = [&](const w4_u4 (&p)[2], int at, int place) {
    unsigned(&w)[8][32] = weights[wave];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) w[i / 4 * 4 + i % 4 / 2 + 2 * half][col] = p[b][i / 2];
      exchanged();
      for (int key = 0; key < 16; ++key) {
        const float x = at_value<XT>(w[key / 2][col], key % 2);
        const bool seen = place + 16 * b + key < sees;
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
          for (int i = 0; i < 4; ++i) {  // dims 32 f + 8 i + 4 half and on
            const at_u2 v = *reinterpret_cast<const at_u2*>(lds + 2 * TILE + at + (16 * b + key) * ROW + (f ^ (ROW == 128 ? key / 2 % 2 : key % 4)) * 64 + i * 16 + half * 8);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float sum = fmaf(x, at_value<XT>(v[j / 2], j % 2), o[f][4 * i + j]);
              o[f][4 * i + j] = seen ? sum : o[f][4 * i + j];
            }
          }
      }
      exchanged();
    }
  };

  // What raised the maximum multiplies the sums a step later, when they have the values of all keys before.
  float factor;
  bool pending = false;
  auto rescale = [&]() {
    if (pending) {
#pragma unroll
      for (int f = 0; f < F; ++f) o[f] *= factor;
      pending = false;
    }
  };
  auto maximum = [&](const at_f16 &s) {
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    const bool high = __any(fmaf(top, scale2, -m) > UP + 8.f);
    if (pending || high) {
      rescale();
      if (high) {
        top = fmaxf(top, __shfl_xor(top, 32));
        const float with = kv_scale_of(top, a.scale2), raised = fmaxf(m, fmaf(top, with, -UP));
        scale2 = raised > m ? with : scale2;
        factor = __builtin_amdgcn_exp2f(m - raised);
        m = raised;
        l *= factor;
        pending = true;
      }
    }
  };
  // pairs first .. last - 1 of the sixteen scores of a row that a lane has
  auto exponentials = [&](const at_f16 &s, w4_u4 (&p)[2], int first, int last) {
#pragma unroll
    for (int i = first; i < last; ++i) {
      const float one = __builtin_amdgcn_exp2f(fmaf(s[2 * i], scale2, -m)), two = __builtin_amdgcn_exp2f(fmaf(s[2 * i + 1], scale2, -m));
      l += one + two;
      p[i / 4][i % 4] = at_pair<XT>(one, two);
    }
  };
  // step j: exponentials of s into p; scores of step j + 1 from keys at `k`, values of step j - 1 at `v`.  All rows see all of step j's keys.  Operands are read from
  // LDS two pairs of products ahead, and a part of the exponentials follows each pair; in this order, to which the compiler is held.
  auto step = [&](at_f16 &s, at_f16 &next, w4_u4 (&p)[2], const w4_u4 (&before)[2], int k, int v) {
    w4_u4 keys[3], values[3];
#pragma unroll
    for (int i = 0; i < 2; ++i) keys[i] = key_piece(k, i), values[i] = value_piece(v, i / F, i % F);
    maximum(s);
    clear_scores(next);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < E; ++i) {  // (E == 2 F)
      if (i + 2 < E) keys[(i + 2) % 3] = key_piece(k, i + 2), values[(i + 2) % 3] = value_piece(v, (i + 2) / F, (i + 2) % F);
      next = at_mfma<XT>(keys[i % 3], q[i], next);
      o[i % F] = at_mfma<XT>(values[i % 3], before[i / F], o[i % F]);
      exponentials(s, p, 8 * i / E, 8 * (i + 1) / E);
      asm volatile("" : "+v"(p[(8 * (i + 1) / E - 1) / 4]), "+v"(l));  // (else they wait for their use, a step later)
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
  };
  // the same where they may not, or where step j or j + 1 may not be the wave's
  auto last_step = [&](int j, at_f16 &s, at_f16 &next, w4_u4 (&p)[2], const w4_u4 (&before)[2], int k, int v, bool seen) {
    if (j < steps) {
      if (j * 32 + 32 > full) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = j * 32 + i / 4 * 8 + i % 4 + 4 * half >= sees ? -INFINITY : s[i];
      }
      maximum(s);
    } else rescale();
    if (j > 0 && j <= steps) {
      if (seen && j * 32 > full) add_seen(before, v, j * 32 - 32);
      else add(before, v);
    }
    if (j + 1 < steps) score(next, k);
    if (j < steps) exponentials(s, p, 0, 8);
  };

  // What is under way when a group begins is there when it ends: the wait is for all of a wave's copies, the barrier for the others'.
  auto arrived = [&]() {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
    __syncthreads();
  };
  if (all > 0) fetch_keys(0), fetch_values(0);
  if (all > kTileKeys) fetch_keys(1);
  arrived();
  if (steps > 0) score(s[0], 0);
  last_step(0, s[0], s[1], p[0], p[1], 32 * ROW, 0, false);
  __syncthreads();
  // group g: steps 2 g + 1 and 2 g + 2, which take keys of tile g + 1 and values of tile g
  int g = 0;
  for (; g < easy; ++g) {
    const int keys = (g + 1) % 2 * TILE, values = g % 2 * TILE;
    if ((g + 2) * kTileKeys < all) fetch_keys(g + 2);
    if ((g + 1) * kTileKeys < all) fetch_values(g + 1);
    step(s[1], s[0], p[1], p[0], keys, values);
    step(s[0], s[1], p[0], p[1], keys + 32 * ROW, values + 32 * ROW);
    arrived();
  }
  for (; g < groups; ++g) {
    const int keys = (g + 1) % 2 * TILE, values = g % 2 * TILE;
    // values that some row may not see: whether one of them is not finite
    bool seen = false;
    if (DP > 128 || least < (g + 1) * kTileKeys) {  // (with more dims the condition has addresses of the loop above spilled: 4096 tokens of 16 heads of 256 254 us, 200 so)
      bool any = false;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const w4_u4 v = *reinterpret_cast<const w4_u4*>(lds + 2 * TILE + values + (i * THREADS + thread) * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) any |= at_odd<XT>(v[j]);
      }
      if (any) odd[g % 2] = 1;
      if (thread == 0) odd[(g + 1) % 2] = 0;  // (which is read no more)
      __syncthreads();
      seen = odd[g % 2];
    }
    if ((g + 2) * kTileKeys < all) fetch_keys(g + 2);
    if ((g + 1) * kTileKeys < all) fetch_values(g + 1);
    last_step(2 * g + 1, s[1], s[0], p[1], p[0], keys, values, seen);
    last_step(2 * g + 2, s[0], s[1], p[0], p[1], keys + 32 * ROW, values + 32 * ROW, seen);
    arrived();
  }
  rescale();

  if constexpr (SPLIT > 1) {
    // the parts' sums come to the first one
    static_assert(SPLIT == 2 && THREADS * F * 64 <= SPLIT * LDS, "one other part, whose sums find room");
    __shared__ float other_m[THREADS], other_l[THREADS];
    float4* to = reinterpret_cast<float4*>(all_lds) + thread;
    if (part) {
      other_m[thread] = m, other_l[thread] = l;
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int i = 0; i < 4; ++i) to[(f * 4 + i) * THREADS] = float4{o[f][4 * i], o[f][4 * i + 1], o[f][4 * i + 2], o[f][4 * i + 3]};
    }
    __syncthreads();
    if (part) return;
    const float high = fmaxf(m, other_m[thread]), here = __builtin_amdgcn_exp2f(m - high), there = __builtin_amdgcn_exp2f(other_m[thread] - high);
    l = fmaf(l, here, other_l[thread] * there);
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 x = to[(f * 4 + i) * THREADS];
        o[f][4 * i] = fmaf(o[f][4 * i], here, x.x * there), o[f][4 * i + 1] = fmaf(o[f][4 * i + 1], here, x.y * there);
        o[f][4 * i + 2] = fmaf(o[f][4 * i + 2], here, x.z * there), o[f][4 * i + 3] = fmaf(o[f][4 * i + 3], here, x.w * there);
      }
  }
  l += __shfl_xor(l, 32);
  const float inverse = l == 0.f ? 0.f : 1.f / l;
  auto result = [&](int f, int i) { return l == 0.f ? 0.f : o[f][i] * inverse; };
  if (a.wide_out) {
    // Rows in pieces of 16 bytes, which come together in LDS, where keys and values (or the parts' sums) have been: a store has whole rows, not 16 bytes of 32 of them.
    char* const to = all_lds + (SPLIT - 1) * LDS + wave * 32 * ROW;
    static_assert(WAVES / SPLIT * 32 * ROW <= LDS, "room for all waves' rows");
    auto place_of = [&](int r, int piece) { return r * ROW + (piece ^ r % (ROW == 128 ? 8 : 16)) * 16; };
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        at_u2 w;
        const float r[4] = {result(f, 4 * i), result(f, 4 * i + 1), result(f, 4 * i + 2), result(f, 4 * i + 3)};
        if (a.out.type == OZ2_BF16) w = at_u2{at_pair<OZ2_BF16>(r[0], r[1]), at_pair<OZ2_BF16>(r[2], r[3])};
        else w = at_u2{at_pair<OZ2_F16>(r[0], r[1]), at_pair<OZ2_F16>(r[2], r[3])};
        *reinterpret_cast<at_u2*>(to + place_of(col, 4 * f + i) + half * 8) = w;
      }
    exchanged();
    constexpr int EACH = 64 / PIECES;  // rows of a store
    const int piece = lane % PIECES;
#pragma unroll
    for (int i = 0; i < 32 / EACH; ++i) {
      const int r = i * EACH + lane / PIECES, row = first_row + r, at = row / a.per_group;
      const int64_t out_at = (tile.begin + at) * a.out.ld_token + ((int64_t)head * a.group + (row - at * a.group)) * a.out.ld_head;
      const w4_u4 w = *reinterpret_cast<const w4_u4*>(to + place_of(r, piece));
      if (row < rows && piece * 8 < a.dim) *reinterpret_cast<w4_u4*>(static_cast<uint16_t*>(a.out.data) + out_at + piece * 8) = w;
    }
    return;
  }
  if (first_row + col >= rows) return;
  const int64_t out_at = (tile.begin + at) * a.out.ld_token + query * a.out.ld_head;
#pragma unroll
  for (int f = 0; f < F; ++f)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = 32 * f + 8 * i + 4 * half;
      if (d >= a.dim) continue;
      float r[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) r[j] = result(f, 4 * i + j);
      if (a.out.type == OZ2_F32)
#pragma unroll
        for (int j = 0; j < 4; ++j) static_cast<float*>(a.out.data)[out_at + d + j] = r[j];
      else if (a.out.type == OZ2_BF16) {
        const at_u2 w = {at_pair<OZ2_BF16>(r[0], r[1]), at_pair<OZ2_BF16>(r[2], r[3])};
        *reinterpret_cast<at_u2*>(static_cast<uint16_t*>(a.out.data) + out_at + d) = w;
      } else {
        const at_u2 w = {at_pair<OZ2_F16>(r[0], r[1]), at_pair<OZ2_F16>(r[2], r[3])};
        *reinterpret_cast<at_u2*>(static_cast<uint16_t*>(a.out.data) + out_at + d) = w;
      }
    }
}

template <int XT, int DP, int WAVES, int SPLIT>
hipError_t oz2_attention_tile_launch(const Attention& a, hipStream_t st) {
  hipLaunchKernelGGL((attention_tile_kernel<XT, DP, WAVES, SPLIT>), dim3((unsigned)(attention_tiles(a, 32 * WAVES / SPLIT) * a.kv_heads)), dim3(64 * WAVES), 0, st, a);
  return hipGetLastError();
}
// (of 129 to 256 values: the sums take half the registers, so four waves; compiled in a file of its own)
template <int XT> hipError_t oz2_attention_wide_of(const Attention& a, hipStream_t st);
template <int XT, int WAVES, int SPLIT>
hipError_t oz2_attention_tile_dims(const Attention& a, hipStream_t st) {
  if (a.dim <= 64) return oz2_attention_tile_launch<XT, 64, WAVES, SPLIT>(a, st);
  if (a.dim <= 96) return oz2_attention_tile_launch<XT, 96, WAVES, SPLIT>(a, st);
  return oz2_attention_tile_launch<XT, 128, WAVES, SPLIT>(a, st);
}
// Tiles of 256 rows read keys least often, and serve sequences that are long on the mean.  Shorter ones: 128 rows, of which two workgroups share a compute unit and
// one begins or ends while the other is at work.  Where even tiles of 128 leave compute units without work, or last much longer than their number needs:
// 128 rows with their keys in two parts.  bf16, causal, 8 query and kv heads of 128 values, us with 256 rows, 128 rows, and parts:
//   sequences          2 x 1024   1 x 2048   1 x 4096   4 x 2048   1 x 8192   24 x 512   3 x 4096   (32 and 8 heads) 12 of 16 to 2000   1 x 4096   1 x 8192
//   256 rows              35         56        100         62        194         44        117                     155                  135        497
//   128 rows              27         43         79         55        174         35        113                     148                  142        511
//   128 rows, parts       25         38         66         58        155         52        133                     204                  162        569
// Few rows: 64 of them with their keys in two parts, of which 65 to 128 dims leave room for one workgroup a compute unit, up to 64 for two.
//   us with 128 rows, 128 in parts, 64 in parts       1 x 512   1 x 1024   1 x 2048   (one head) 1 x 4096   1 x 16384   4 x 512   8 x 512
//   8 heads of 128 values                            17 17 15   26 24 20   42 36 31           74 59 48     269 206 167  18 18 16  20 20 26
//   8 heads of 64                                    13 12 11   19 16 14   30 24 21           53 40 33     191 135 108  13 13 11  14 13 13
template <int XT>
hipError_t oz2_attention_tile_of(const Attention& a, hipStream_t st) {
  if (a.dim > 128) return oz2_attention_wide_of<XT>(a, st);
  const int64_t tiles = a.tokens * a.heads / 256, mean = a.tokens / a.sequences;
  if (mean >= 500 && tiles <= (a.dim <= 64 ? 128 : 64)) return oz2_attention_tile_dims<XT, 4, 2>(a, st);
  if (mean >= 3000 ? tiles <= 288 : mean >= 1000 && tiles <= 128) return oz2_attention_tile_dims<XT, 8, 2>(a, st);
  return mean >= 3000 ? oz2_attention_tile_dims<XT, 8, 1>(a, st) : oz2_attention_tile_dims<XT, 4, 1>(a, st);
}

#endif
#endif
