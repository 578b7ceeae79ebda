// Attention of a few new tokens over a cache held in 4 bits (oz2_kv4_attention): the kernel of one type of query.
//
// A workgroup has a chunk of places of one sequence and kv head; its four waves take tiles of 32 places in turn, and sixteen rows (pairs of a new token and
// one of the kv head's query heads) at a time.  For a tile, with c the codes of a key or value, s and o its scale and offset:
//   t = s sum_d q_d c_d + o sum_d q_d,    p = exp2(scale log2(e) t - m),    numerator_d = sum p s c_d + sum p o,    denominator = sum p
// Codes go to the matrix cores as they lie in a word, where the bits of a bf16 below 2^-125 count in steps of 2^-133 from 0 on, with and without an exponent: four
// bits at the bottom of a half word are c 2^-133, the four above them c 2^-129, and an AND makes operands of two codes.  q is taken times 2^64 (2^60 where
// it meets the latter) and p times 2^80, so that sums are far from either end of FP32; the powers of two come off again in `scale2` and at the end.
// Nothing has to be added to a code and taken off later.  (FP32 results would show that the matrix cores cut sums off instead of rounding them, in
// proportion to the sums of codes, which lie on one side of 0: for them operands are 2 (c - 7.5), at four instructions a pair, and the offsets o + 7.5 s.)  q is
// made of one bf16 (bf16), two (f16) or three (f32) exactly, p s of two bf16, or three for FP32 results: an error of 2^-16 or 2^-24 of it.
// The products are keys x rows and then dims x rows, so that every lane has one row throughout: what the first product leaves in a lane (four places of each
// half of the tile) is what it needs as its part of the second's operand, and maxima and sums stay in lanes until the end.  m is raised only
// where a score is more than 8 above it (to base 2).
// Nothing goes through LDS but the four waves' results.  A lane reads of keys the codes of one place (a quarter of the row), of values those of eight places
// (a sixteenth of each row): a tile's words are in registers before the previous tile is done with.
//   Bound by the bytes of the cache where sequences are long: 64 of 2048 to 32768 places, 8 kv heads of 128, BF16, are read at 4.8 TB/s (163 to 180 us, where a copy
// moves 5.0); with FP16 queries, whose second term doubles the first products, and 16 of 2000 to 8192 places, 3 TB/s (29 us).
#ifndef OZ2_KV4_STEP_H
#define OZ2_KV4_STEP_H

#include "oz2_kv4.h"
#include "oz2_fast_div.h"
#include "oz2_w4_core.h"

#ifdef __HIPCC__

constexpr int kStepRows = 16, kStepTile = 32, kStepWaves = 4;

struct Kv4Step {
  oz2_kv4_cache c;
  oz2_kv4_sequences on;
  oz2_rows q, out;
  int heads, group, dim, capacity, page_size, chunk;
  FastDiv per_page, per_group;
  float scale2;  // scale log2(e) over the factor of the scores
  // of (chunk, row) and, of scores, (row, place); rows are those of q, (token, head)
  float *part, *stats, *scores;
  int64_t rows;
};

template <int XT> constexpr int step_parts() { return XT == OZ2_BF16 ? 1 : XT == OZ2_F16 ? 2 : 3; }

__device__ __forceinline__ unsigned bf16_pair(float a, float b) {
  typedef float Two __attribute__((ext_vector_type(2)));
  typedef __bf16 Brain __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_convertvector((Two{a, b}), Brain));
}
// the bf16 values of a pair, taken off: what is left of a and b for the next term
__device__ __forceinline__ unsigned bf16_term(float& a, float& b) {
  const unsigned w = bf16_pair(a, b);
  a -= __uint_as_float(w << 16), b -= __uint_as_float(w & 0xffff0000u);
  return w;
}
// codes j and j + 4 of a word as bf16 in steps of 2^-133: c itself (j odd: 16 c), or 2 (c - 7.5) = +- (2 m + 1) of a word whose codes step_centred has made
// (sign, m)
template <bool CENTRED>
__device__ __forceinline__ unsigned code_pair(unsigned w, int j) {
  if constexpr (!CENTRED) return (j < 2 ? w : w >> 8) & (j % 2 ? 0x00f000f0u : 0x000f000fu);
  else return ((j == 0 ? w << 1 : w >> (4 * j - 1)) & 0x000e000eu) | 0x00010001u | (w << (12 - 4 * j) & 0x80008000u);
}
__device__ __forceinline__ unsigned step_centred(unsigned w) {
  const unsigned sign = ~w & 0x88888888u;
  return ((w & 0x77777777u) ^ (sign - (sign >> 3))) | sign;
}
constexpr float kStepUp = 0x1p64f, kStepFactor = 0x1p80f;  // of q, and of p
// what brings sums of q c and of p s c back: operands come in steps of 2^-133, or twice that
template <int XT> constexpr bool step_is_centred() { return XT == OZ2_F32; }
template <int XT> constexpr float step_score() { return step_is_centred<XT>() ? 0x1p68f : 0x1p69f; }
template <int XT> constexpr float step_back() { return step_is_centred<XT>() ? 0x1p52f : 0x1p53f; }
__device__ __forceinline__ w4_f4 step_mfma(w4_u4 a, w4_u4 b, w4_f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(w4_bf8, a), __builtin_bit_cast(w4_bf8, b), c, 0, 0, 0);
}
// Loads of 4, 8 or 16 bytes at `at` bytes, 32 bits of a lane's own, behind a base that is the same for all lanes: no address is formed by the vector units.
typedef __amdgpu_buffer_rsrc_t StepBase;
__device__ __forceinline__ StepBase step_base(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, -1, 0x00027000);
}
template <int N>
__device__ __forceinline__ void step_load(StepBase base, unsigned at, unsigned (&w)[N]) {
  if constexpr (N == 1) w[0] = __builtin_amdgcn_raw_buffer_load_b32(base, at, 0, 0);
  else if constexpr (N == 2) {
    const auto x = __builtin_amdgcn_raw_buffer_load_b64(base, at, 0, 0);
    w[0] = x[0], w[1] = x[1];
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const auto x = __builtin_amdgcn_raw_buffer_load_b128(base, at + 16 * i, 0, 0);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[4 * i + j] = x[j];
    }
  }
}
// (fmaxf has its operands made quiet first, an instruction each)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ float half_of(unsigned w, int upper) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(upper ? w >> 16 : w)); }

// DP: dim rounded up to 64, 128 or 256
template <int DP>
struct StepTile {
  unsigned k[2][DP / 32];    // a quarter of a row of keys, of each half of the tile
  unsigned v[8][(DP + 127) / 128];  // a sixteenth of the rows of eight values: places 4 quarter + i of each half
  w4_u4 ks[2], vs[2];        // scale and offset of these
  bool there[2];
};

template <int XT, int DP, bool WIDE>
__global__ void __launch_bounds__(256, XT != OZ2_F32 && DP <= 128 ? 3 : 1) kv4_step_kernel(Kv4Step a) {
  constexpr int E = DP / 32, F = DP / 16, PARTS = step_parts<XT>(), TERMS = XT == OZ2_F32 ? 3 : 2;
  // p's factor comes with the exponent, for which that has seven bits less: 2^-18 of p, which FP32 results would show; there p s is multiplied by it
  __shared__ float merged[kStepWaves][kStepRows][DP + 1];
  __shared__ float merged_m[kStepWaves][kStepRows], merged_l[kStepWaves][kStepRows], merged_c[kStepWaves][kStepRows];
  constexpr bool CENTRED = step_is_centred<XT>();
  constexpr float SHIFT = XT == OZ2_F32 ? 0.f : 80.f;
  const int head = blockIdx.x, s = blockIdx.y, lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int col = lane % 16, quarter = lane / 16;
  const KvRange r = kv_range(a.on.cu, s, a.on.tokens);
  const int news = (int)(r.end - r.begin), rows = news * a.group;
  const int held = kv_held(a.on.lengths, s, a.capacity);
  const int c0 = blockIdx.z * a.chunk;
  if (rows == 0 || (c0 >= held && c0 > 0)) return;
  const int c1 = min(held, c0 + a.chunk);
  const bool whole = held <= a.chunk;
  // (read by scalar loads: a vector load would have to be waited for, and with it the tiles that were asked for before)
  typedef const int32_t __attribute__((address_space(4)))* Scalars;
  const Scalars table = (Scalars)(uintptr_t)(a.on.table + s * a.on.ld_table);

  const int64_t codes_head = head * a.c.codes_head, scales_head = head * a.c.scales_head;
  const int bytes = WIDE ? DP / 2 : a.dim / 2;
  // where a lane's words are among sixteen rows; words past a row's end are read from its start, and meet zeros of q or are not stored
  unsigned k_at[WIDE ? 1 : E], v_at[WIDE ? 1 : (DP + 127) / 128];
  for (int e = 0; e < (WIDE ? 1 : E); ++e) {
    const int word = WIDE ? quarter * E : e * 4 + quarter;
    k_at[e] = col * bytes + (word * 4 < bytes ? word * 4 : 0);
  }
  for (int u = 0; u < (WIDE ? 1 : (DP + 127) / 128); ++u) v_at[u] = quarter * 4 * bytes + (col * (DP / 32) + 4 * u < bytes ? col * (DP / 32) + 4 * u : 0);
  const unsigned s_at = quarter * 16;

  struct Pages { int id[2]; };
  auto pages = [&](int tile) {
    Pages p;
    for (int i = 0; i < 2; ++i) {
      const int place = tile * kStepTile + 16 * i;
      const int id = table[(place < c1 ? place : c0) / a.per_page];
      p.id[i] = place < c1 && id >= 0 && id < a.c.pages ? id : -1;
    }
    return p;
  };
  auto fetch = [&](int tile, const Pages& p) {
    StepTile<DP> r;
    for (int i = 0; i < 2; ++i) {
      const int place = tile * kStepTile + 16 * i, in = p.id[i] < 0 ? 0 : place - place / a.per_page * a.page_size;
      const int64_t page = p.id[i] < 0 ? 0 : p.id[i];
      r.there[i] = p.id[i] >= 0;
      const int64_t codes = page * a.c.codes_page + codes_head + (int64_t)in * bytes, scales = page * a.c.scales_page + scales_head + in;
      const StepBase k = step_base(a.c.k_codes + codes), v = step_base(a.c.v_codes + codes);
      if constexpr (WIDE) step_load(k, k_at[0], r.k[i]);
      else {
#pragma unroll
        for (int e = 0; e < E; ++e) r.k[i][e] = __builtin_amdgcn_raw_buffer_load_b32(k, k_at[e], 0, 0);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (DP == 64) r.v[4 * i + j][0] = __builtin_amdgcn_raw_buffer_load_b16(v, v_at[0] + j * bytes, 0, 0);
        else if constexpr (WIDE) step_load(v, v_at[0] + j * bytes, r.v[4 * i + j]);
        else {
#pragma unroll
          for (int u = 0; u < DP / 128; ++u) r.v[4 * i + j][u] = __builtin_amdgcn_raw_buffer_load_b32(v, v_at[u] + j * bytes, 0, 0);
        }
      }
      r.ks[i] = __builtin_bit_cast(w4_u4, __builtin_amdgcn_raw_buffer_load_b128(step_base(static_cast<const unsigned*>(a.c.k_scales) + scales), s_at, 0, 0));
      r.vs[i] = __builtin_bit_cast(w4_u4, __builtin_amdgcn_raw_buffer_load_b128(step_base(static_cast<const unsigned*>(a.c.v_scales) + scales), s_at, 0, 0));
    }
    return r;
  };

  for (int r0 = 0; r0 < rows; r0 += kStepRows) {
    const int row = r0 + col, fresh = min(row, rows - 1) / a.per_group;
    const int64_t token = r.begin + fresh, query = (int64_t)head * a.group + (min(row, rows - 1) - fresh * a.group);
    const int sees = held - news + fresh + 1;  // places
    w4_u4 q[PARTS][E];
    float sum = 0.f;
    for (int e = 0; e < E; ++e) {
      const int word = WIDE ? quarter * E + e : e * 4 + quarter;
      float x[8] = {};
      if (word * 8 < a.dim) kv_load8<XT>(a.q.data, token * a.q.ld_token + query * a.q.ld_head + word * 8, x);
      for (int j = 0; j < 8; ++j) {
        sum += x[j];
        x[j] *= !CENTRED && j % 2 ? kStepUp / 16 : kStepUp;
      }
      for (int t = 0; t < PARTS; ++t)
        for (int j = 0; j < 4; ++j) q[t][e][j] = bf16_term(x[j], x[j + 4]);
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    sum *= 1.f / step_score<XT>();

    float m = kNoScore, l = 0.f, c = 0.f;  // (finite, so that nothing that is not seen becomes a NaN)
    w4_f4 o[F];
    for (int f = 0; f < F; ++f) o[f] = w4_f4{0.f, 0.f, 0.f, 0.f};

    // a tile's places: `cut` where some are hidden from some row
    auto take = [&](int tile, StepTile<DP>& now) {
      const int begin = tile * kStepTile;
      const bool cut = begin + kStepTile > held - news || begin + kStepTile > c1 || !now.there[0] || !now.there[1];
      unsigned hidden = 0;
      if (cut) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int place = begin + i / 4 * 16 + quarter * 4 + i % 4;
          const bool hides = place >= sees || place >= c1 || !now.there[i / 4];
          hidden |= hides ? 1u << i : 0u;
          // (what is there may be a NaN)
          now.ks[i / 4][i % 4] = hides ? 0u : now.ks[i / 4][i % 4];
          now.vs[i / 4][i % 4] = hides ? 0u : now.vs[i / 4][i % 4];
        }
      }
      float t[8];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        w4_f4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < E; ++e) {
          w4_u4 k;
          const unsigned word = CENTRED ? step_centred(now.k[i][e]) : now.k[i][e];
#pragma unroll
          for (int j = 0; j < 4; ++j) k[j] = code_pair<CENTRED>(word, j);
#pragma unroll
          for (int x = 0; x < PARTS; ++x) acc = step_mfma(k, q[x][e], acc);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) t[4 * i + j] = fmaf(half_of(now.ks[i][j], 0), acc[j], (CENTRED ? fmaf(7.5f, half_of(now.ks[i][j], 0), half_of(now.ks[i][j], 1)) * sum
                                                                           : fmaf(half_of(now.ks[i][j], 1), sum, 0.f)));  // (+ 0: one instruction that takes FP16)
      }
      if (cut) {
        asm volatile("" : "+v"(hidden));  // (a branch: eight selects by conditions that hardly ever hold cost more)
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = hidden >> i & 1 ? -INFINITY : t[i];
      }
      if (a.scores && row < rows) {
        float* to = a.scores + (token * a.heads + query) * a.capacity;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int place = begin + i / 4 * 16 + quarter * 4 + i % 4;
          if (place < c1) to[place] = t[i];
        }
      }
      const float top = max3(max3(max3(t[0], t[1], t[2]), t[3], t[4]), max3(t[5], t[6], t[7]), t[7]);
      // (a row of large scores, and one without any: m is taken off ahead of the exponent, where SHIFT would be lost in it)
      float shift = SHIFT - (fabsf(m) > kLarge ? 0.f : m);
      if (__any(fabsf(m) > kLarge || fmaf(top, a.scale2, shift) > SHIFT + 8.f)) {
        float high = fmaxf(top, __shfl_xor(top, 16));
        high = fmaxf(high, __shfl_xor(high, 32));
        const float raised = fmaxf(m, high * kv_scale_of(high, a.scale2)), f = __builtin_amdgcn_exp2f(m - raised);
        m = raised;
        l *= f, c *= f;
#pragma unroll
        for (int i = 0; i < F; ++i) o[i] *= f;
        const bool large = fabsf(m) > kLarge;
        const float above = kv_power_above(a.scale2), back = __builtin_amdgcn_rcpf(a.scale2);
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = large ? fmaf(t[i], above, -m) * back : t[i];
        shift = SHIFT - (large ? 0.f : m);
      }
      float w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = __builtin_amdgcn_exp2f(fmaf(t[i], a.scale2, shift));
        l += p;
        w[i] = fmaf(p, half_of(now.vs[i / 4][i % 4], 0), 0.f);
        if constexpr (XT == OZ2_F32) w[i] *= kStepFactor;
        const float shift = half_of(now.vs[i / 4][i % 4], 1);
        c = fmaf(p, CENTRED ? fmaf(7.5f, half_of(now.vs[i / 4][i % 4], 0), shift) : shift, c);
      }
      w4_u4 b[TERMS];
#pragma unroll
      for (int x = 0; x < TERMS; ++x)
#pragma unroll
        for (int j = 0; j < 4; ++j) b[x][j] = bf16_term(w[2 * j], w[2 * j + 1]);
#pragma unroll
      for (int u = 0; u < (DP + 127) / 128; ++u) {
        unsigned low[4], high[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          low[j] = __builtin_amdgcn_perm(now.v[2 * j + 1][u], now.v[2 * j][u], 0x05040100);
          high[j] = __builtin_amdgcn_perm(now.v[2 * j + 1][u], now.v[2 * j][u], 0x07060302);
          if constexpr (CENTRED) low[j] = step_centred(low[j]), high[j] = step_centred(high[j]);
        }
#pragma unroll
        for (int e = 0; e < (DP == 64 ? 4 : 8); ++e) {
          w4_u4 v;
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = code_pair<CENTRED>(e < 4 ? low[j] : high[j], e % 4);
#pragma unroll
          for (int x = 0; x < TERMS; ++x) o[u * 8 + e] = step_mfma(v, b[x], o[u * 8 + e]);
        }
      }
    };

    const int first = c0 / kStepTile + wave, last = (c1 + kStepTile - 1) / kStepTile;
    if (first < last) {
      Pages p = pages(first);
      StepTile<DP> one = fetch(first, p), two;
      p = pages(first + kStepWaves);
      for (int tile = first;; tile += 2 * kStepWaves) {
        two = fetch(tile + kStepWaves, p);
        p = pages(tile + 2 * kStepWaves);
        take(tile, one);
        if (tile + kStepWaves >= last) break;
        one = fetch(tile + 2 * kStepWaves, p);
        p = pages(tile + 3 * kStepWaves);
        take(tile + kStepWaves, two);
        if (tile + 2 * kStepWaves >= last) break;
      }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    c += __shfl_xor(c, 16);
    c += __shfl_xor(c, 32);
    if constexpr (XT != OZ2_F32) l *= 1.f / kStepFactor, c *= 1.f / kStepFactor;

    // the waves' results together
    __syncthreads();
    if (quarter == 0) merged_m[wave][col] = m, merged_l[wave][col] = l, merged_c[wave][col] = c;
    for (int f = 0; f < F; ++f)
      for (int i = 0; i < 4; ++i) merged[wave][col][(quarter * 4 + i) * F + f] = o[f][i] * (!CENTRED && f % 2 ? step_back<XT>() / 16 : step_back<XT>());
    __syncthreads();
    for (int at = threadIdx.x; at < kStepRows * (DP / 8); at += 256) {
      const int b = at / (DP / 8), d = at % (DP / 8) * 8;
      if (r0 + b >= rows || d >= a.dim) continue;
      float high = merged_m[0][b], factor[kStepWaves], total = 0.f, shift = 0.f, v[8] = {};
      for (int i = 1; i < kStepWaves; ++i) high = fmaxf(high, merged_m[i][b]);
      for (int i = 0; i < kStepWaves; ++i) {
        factor[i] = __builtin_amdgcn_exp2f(merged_m[i][b] - high);
        total = fmaf(factor[i], merged_l[i][b], total);
        shift = fmaf(factor[i], merged_c[i][b], shift);
      }
      for (int j = 0; j < 8; ++j) {
        v[j] = shift;
        for (int i = 0; i < kStepWaves; ++i) v[j] = fmaf(factor[i], merged[i][b][d + j], v[j]);
      }
      const int of = (r0 + b) / a.per_group;
      const int64_t token = r.begin + of, query = (int64_t)head * a.group + (r0 + b - of * a.group), row = token * a.heads + query;
      if (whole) {
        for (int j = 0; j < 8; ++j) w4_store(a.out.type, a.out.data, token * a.out.ld_token + query * a.out.ld_head + d + j, total == 0.f ? 0.f : v[j] / total);
      } else {
        float* to = a.part + ((int64_t)blockIdx.z * a.rows + row) * a.dim + d;
        for (int j = 0; j < 8; ++j) to[j] = v[j];
      }
      if (d == 0 && a.stats) {
        float* to = a.stats + ((int64_t)blockIdx.z * a.rows + row) * 2;
        to[0] = high, to[1] = total;
      }
    }
    __syncthreads();
  }
}

template <int XT>
hipError_t oz2_kv4_step_of(const Kv4Step& a, dim3 grid, hipStream_t st) {
  const dim3 block(256);
  if (a.dim == 64) hipLaunchKernelGGL((kv4_step_kernel<XT, 64, true>), grid, block, 0, st, a);
  else if (a.dim < 64) hipLaunchKernelGGL((kv4_step_kernel<XT, 64, false>), grid, block, 0, st, a);
  else if (a.dim == 128) hipLaunchKernelGGL((kv4_step_kernel<XT, 128, true>), grid, block, 0, st, a);
  else if (a.dim < 128) hipLaunchKernelGGL((kv4_step_kernel<XT, 128, false>), grid, block, 0, st, a);
  else if (a.dim == 256) hipLaunchKernelGGL((kv4_step_kernel<XT, 256, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((kv4_step_kernel<XT, 256, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

#endif
#endif
