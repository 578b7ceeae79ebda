// Attention of a few new tokens over a cache held in 4 bits (oz2_kv4_attention): the kernel of one type of query.
//
// A workgroup has a chunk of places of one sequence and kv head; its four waves take tiles of 32 places in turn, and sixteen rows (pairs of a new token and
// one of the kv head's query heads) at a time.  For a tile, with c the codes of a key or value, s and o its scale and offset:
//   t = s sum_d q_d c_d + o sum_d q_d,    p = exp2(scale log2(e) t - m),    numerator_d = sum p s c_d + sum p o,    denominator = sum p
// Codes go to the matrix cores as bf16 16 + c (bits put under an exponent: a shift and an and-or for two); the 16 comes off again as -16 sum q (what the
// sums start from) and -16 sum p s.  q is made of one bf16 (bf16), two (f16) or three (f32) exactly, p s of two bf16, or three for FP32 results: an error of 2^-17 or
// 2^-25 of it.
// The products are keys x rows and then dims x rows, so that every lane has one row throughout: what the first product leaves in a lane (four places of each
// half of the tile) is what it needs as its part of the second's operand, and maxima and sums stay in lanes until the end.  m is raised only
// where a score is more than 2^8 above it.
// Nothing goes through LDS but the four waves' results.  A lane reads of keys the codes of one place (a quarter of the row), of values those of eight places
// (a sixteenth of each row): a tile's words are in registers before the previous tile is done with.
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
  float scale2;  // scale log2(e)
  // of (chunk, row) and, of scores, (row, place); rows are those of q, (token, head)
  float *part, *stats, *scores;
  int64_t rows;
};

template <int XT> constexpr int step_parts() { return XT == OZ2_BF16 ? 1 : XT == OZ2_F16 ? 2 : 3; }

__device__ __forceinline__ unsigned bf16_pair(float a, float b) {
  return __builtin_bit_cast(uint16_t, (__bf16)a) | (unsigned)__builtin_bit_cast(uint16_t, (__bf16)b) << 16;
}
// the bf16 values of a pair, taken off: what is left of a and b for the next term
__device__ __forceinline__ unsigned bf16_term(float& a, float& b) {
  const unsigned w = bf16_pair(a, b);
  a -= __uint_as_float(w << 16), b -= __uint_as_float(w & 0xffff0000u);
  return w;
}
// codes j and j + 4 of a word as a pair of bf16 16 + c
__device__ __forceinline__ unsigned code_pair(unsigned w, int j) {
  return ((j == 0 ? w << 3 : w >> (4 * j - 3)) & 0x00780078u) | 0x41804180u;
}
__device__ __forceinline__ w4_f4 step_mfma(w4_u4 a, w4_u4 b, w4_f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(w4_bf8, a), __builtin_bit_cast(w4_bf8, b), c, 0, 0, 0);
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
__global__ void __launch_bounds__(256) kv4_step_kernel(Kv4Step a) {
  constexpr int E = DP / 32, F = DP / 16, PARTS = step_parts<XT>(), TERMS = XT == OZ2_F32 ? 3 : 2;
  __shared__ float merged[kStepWaves][kStepRows][DP + 1];
  __shared__ float merged_m[kStepWaves][kStepRows], merged_l[kStepWaves][kStepRows], merged_c[kStepWaves][kStepRows];
  const int head = blockIdx.y, s = blockIdx.z, lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int col = lane % 16, quarter = lane / 16;
  const KvRange r = kv_range(a.on.cu, s, a.on.tokens);
  const int news = (int)(r.end - r.begin), rows = news * a.group;
  const int held = kv_held(a.on.lengths, s, a.capacity);
  const int c0 = blockIdx.x * a.chunk;
  if (rows == 0 || (c0 >= held && c0 > 0)) return;
  const int c1 = min(held, c0 + a.chunk);
  const bool whole = held <= a.chunk;
  const int32_t* table = a.on.table + s * a.on.ld_table;

  const int64_t codes_head = head * a.c.codes_head, scales_head = head * a.c.scales_head;
  const int bytes = a.dim / 2;
  // where a lane's words are in a row; words past its end are read from its start, and meet zeros of q or are not stored
  int k_at[E];
  for (int e = 0; e < E; ++e) {
    const int word = WIDE ? quarter * E + e : e * 4 + quarter;
    k_at[e] = word * 4 < bytes ? word * 4 : 0;
  }
  int v_at[(DP + 127) / 128];
  for (int u = 0; u < (DP + 127) / 128; ++u) v_at[u] = col * (DP / 32) + 4 * u < bytes ? col * (DP / 32) + 4 * u : 0;

  struct Pages { int id[2]; };
  auto pages = [&](int tile) {
    Pages p;
    for (int i = 0; i < 2; ++i) {
      const int place = tile * kStepTile + 16 * i;
      const int at = place < c1 ? place : c0;
      const int id = __builtin_amdgcn_readfirstlane(place < c1 ? table[at / a.per_page] : -1);
      p.id[i] = id >= 0 && id < a.c.pages ? id : -1;
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
      const uint8_t* k = a.c.k_codes + codes;
      const uint8_t* v = a.c.v_codes + codes;
      if constexpr (WIDE) {
        struct __attribute__((packed, aligned(4))) Words { unsigned w[E]; };
        const Words w = *reinterpret_cast<const Words*>(k + col * bytes + quarter * (E * 4));
        for (int e = 0; e < E; ++e) r.k[i][e] = w.w[e];
      } else {
        for (int e = 0; e < E; ++e) r.k[i][e] = *reinterpret_cast<const unsigned*>(k + col * bytes + k_at[e]);
      }
      for (int j = 0; j < 4; ++j) {
        const uint8_t* at = v + (quarter * 4 + j) * bytes;
        if constexpr (DP == 64) r.v[4 * i + j][0] = *reinterpret_cast<const uint16_t*>(at + v_at[0]);
        else if constexpr (WIDE) {
          struct __attribute__((packed, aligned(4))) Words { unsigned w[DP / 128]; };
          const Words w = *reinterpret_cast<const Words*>(at + v_at[0]);
          for (int u = 0; u < DP / 128; ++u) r.v[4 * i + j][u] = w.w[u];
        } else {
          for (int u = 0; u < DP / 128; ++u) r.v[4 * i + j][u] = *reinterpret_cast<const unsigned*>(at + v_at[u]);
        }
      }
      r.ks[i] = *reinterpret_cast<const w4_u4*>(static_cast<const unsigned*>(a.c.k_scales) + scales + quarter * 4);
      r.vs[i] = *reinterpret_cast<const w4_u4*>(static_cast<const unsigned*>(a.c.v_scales) + scales + quarter * 4);
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
      for (int j = 0; j < 8; ++j) sum += x[j];
      for (int t = 0; t < PARTS; ++t)
        for (int j = 0; j < 4; ++j) q[t][e][j] = bf16_term(x[j], x[j + 4]);
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);

    float m = -3e38f, l = 0.f, c = 0.f;  // m: finite, so that nothing that is not seen becomes a NaN
    w4_f4 o[F];
    for (int f = 0; f < F; ++f) o[f] = w4_f4{0.f, 0.f, 0.f, 0.f};

    const int first = c0 / kStepTile + wave, last = (c1 + kStepTile - 1) / kStepTile;
    if (first < last) {
      Pages p = pages(first);
      StepTile<DP> next = fetch(first, p);
      p = pages(first + kStepWaves);
      for (int tile = first; tile < last; tile += kStepWaves) {
        const StepTile<DP> now = next;
        next = fetch(tile + kStepWaves, p);
        p = pages(tile + 2 * kStepWaves);

        float t[8];
        for (int i = 0; i < 2; ++i) {
          w4_f4 acc = {-16.f * sum, -16.f * sum, -16.f * sum, -16.f * sum};
          for (int e = 0; e < E; ++e) {
            w4_u4 k;
            for (int j = 0; j < 4; ++j) k[j] = code_pair(now.k[i][e], j);
            for (int x = 0; x < PARTS; ++x) acc = step_mfma(k, q[x][e], acc);
          }
          for (int j = 0; j < 4; ++j) t[4 * i + j] = fmaf(half_of(now.ks[i][j], 0), acc[j], half_of(now.ks[i][j], 1) * sum);
        }
        const bool cut = tile * kStepTile + kStepTile > held - news || tile * kStepTile + kStepTile > c1 || !now.there[0] || !now.there[1];
        bool hidden[8] = {};
        if (cut) {
          for (int i = 0; i < 8; ++i) {
            const int place = tile * kStepTile + i / 4 * 16 + quarter * 4 + i % 4;
            hidden[i] = place >= sees || place >= c1 || !now.there[i / 4];
            if (hidden[i]) t[i] = -INFINITY;
          }
        }
        if (a.scores && row < rows) {
          float* to = a.scores + (token * a.heads + query) * a.capacity;
          for (int i = 0; i < 8; ++i) {
            const int place = tile * kStepTile + i / 4 * 16 + quarter * 4 + i % 4;
            if (place < c1) to[place] = t[i];
          }
        }
        float x[8], top = -INFINITY;
        for (int i = 0; i < 8; ++i) {
          x[i] = fmaf(t[i], a.scale2, -m);
          top = fmaxf(top, x[i]);
        }
        if (__any(top > 8.f)) {
          float high = -INFINITY;
          for (int i = 0; i < 8; ++i) high = fmaxf(high, t[i] * a.scale2);
          high = fmaxf(high, __shfl_xor(high, 16));
          high = fmaxf(high, __shfl_xor(high, 32));
          const float raised = fmaxf(m, high), f = __builtin_amdgcn_exp2f(m - raised);
          m = raised;
          l *= f, c *= f;
          for (int i = 0; i < F; ++i) o[i] *= f;
          for (int i = 0; i < 8; ++i) x[i] = fmaf(t[i], a.scale2, -m);
        }
        float w[8];
        for (int i = 0; i < 8; ++i) {
          const float p = __builtin_amdgcn_exp2f(x[i]);
          l += p;
          w[i] = p * half_of(now.vs[i / 4][i % 4], 0);
          float shift = p * half_of(now.vs[i / 4][i % 4], 1);
          if (cut && hidden[i]) w[i] = shift = 0.f;
          c += fmaf(-16.f, w[i], shift);
        }
        w4_u4 b[TERMS];
        for (int x = 0; x < TERMS; ++x)
          for (int j = 0; j < 4; ++j) b[x][j] = bf16_term(w[2 * j], w[2 * j + 1]);
        for (int u = 0; u < (DP + 127) / 128; ++u) {
          unsigned low[4], high[4];
          for (int j = 0; j < 4; ++j) {
            low[j] = __builtin_amdgcn_perm(now.v[2 * j + 1][u], now.v[2 * j][u], 0x05040100);
            high[j] = __builtin_amdgcn_perm(now.v[2 * j + 1][u], now.v[2 * j][u], 0x07060302);
          }
          for (int e = 0; e < (DP == 64 ? 4 : 8); ++e) {
            w4_u4 v;
            for (int j = 0; j < 4; ++j) v[j] = code_pair(e < 4 ? low[j] : high[j], e % 4);
            for (int x = 0; x < TERMS; ++x) o[u * 8 + e] = step_mfma(v, b[x], o[u * 8 + e]);
          }
        }
      }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    c += __shfl_xor(c, 16);
    c += __shfl_xor(c, 32);

    // the waves' results together
    __syncthreads();
    if (quarter == 0) merged_m[wave][col] = m, merged_l[wave][col] = l, merged_c[wave][col] = c;
    for (int f = 0; f < F; ++f)
      for (int i = 0; i < 4; ++i) merged[wave][col][(quarter * 4 + i) * F + f] = o[f][i];
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
        float* to = a.part + ((int64_t)blockIdx.x * a.rows + row) * a.dim + d;
        for (int j = 0; j < 8; ++j) to[j] = v[j];
      }
      if (d == 0 && a.stats) {
        float* to = a.stats + ((int64_t)blockIdx.x * a.rows + row) * 2;
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
