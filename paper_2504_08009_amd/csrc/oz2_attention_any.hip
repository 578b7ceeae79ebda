// Attention over packed prompts for any type, dim up to 256 and strides, in FP32 throughout.
//
// A workgroup has 32 rows; its four waves take tiles of 32 keys in turn, each with sums and a maximum of its own, which come together at the end.  Products are
// keys x rows and dims x rows on the FP32 matrix cores (32 x 32 x 2), so that a lane has one row throughout, and what it holds of the first product is what the
// second one wants of it: places 8 (i / 4) + i % 4 and, in the upper half of the lanes, four further on.  Keys and values are read by the lanes that need
// them, from the caches, a few products ahead: so two waves fit a SIMD with 128 dims, three with 64.  m follows the maximum only where a score is more than 8 above it (to base 2).
//   The matrix cores bound it where it is long: 4096 tokens of 16 query and 4 kv heads in FP32, causal, take 648 us with 128 dims (106 TFLOP/s; a large matrix product
// reaches 153), 343 with 64 (100; exponentials are more of it), 2010 with 256 (68; one wave a SIMD).  Few rows are bound by the tiles' number: a compute unit that
// gets two where others have one takes twice as long.
#include "oz2_attention.h"

#include <type_traits>

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));
constexpr int kRows = 32, kKeys = 32;

// Four values beside each other as they are read, made FP32 where they are used: so that no load is waited for before.  FOURS: by one load, of rows whose dim is a
// multiple of four.
template <int XT, bool FOURS>
struct Four {
  unsigned w[FOURS && XT != OZ2_F32 ? 2 : 4];
  __device__ __forceinline__ void read(const char* row, int d, int dim) {
    if constexpr (!FOURS) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = one(row, d + j < dim ? d + j : 0);
    } else {
      struct __attribute__((packed, aligned(XT == OZ2_F32 ? 4 : 2))) Words { unsigned w[XT == OZ2_F32 ? 4 : 2]; };
      const Words x = *reinterpret_cast<const Words*>(row + (d < dim ? d : 0) * (XT == OZ2_F32 ? 4 : 2));
#pragma unroll
      for (int j = 0; j < (XT == OZ2_F32 ? 4 : 2); ++j) w[j] = x.w[j];
    }
  }
  static __device__ __forceinline__ unsigned one(const char* row, int d) {
    if constexpr (XT == OZ2_F32) return reinterpret_cast<const unsigned*>(row)[d];
    else return reinterpret_cast<const uint16_t*>(row)[d];
  }
  static __device__ __forceinline__ float value(unsigned w) {
    if constexpr (XT == OZ2_F32) return __uint_as_float(w);
    else if constexpr (XT == OZ2_BF16) return __uint_as_float(w << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)w);
  }
  __device__ __forceinline__ float operator[](int j) const {
    if constexpr (FOURS && XT != OZ2_F32) return value(j % 2 ? w[j / 2] >> 16 : w[j / 2] & 0xffff);
    else return value(w[j]);
  }
};

template <int XT, int DP, bool FOURS>
__global__ void __launch_bounds__(256, DP <= 64 ? 3 : DP <= 128 ? 2 : 1) attention_any_kernel(Attention a) {
  constexpr int E = DP / 8, F = DP / 32, SIZE = XT == OZ2_F32 ? 4 : 2;
  constexpr int AHEAD = 4;  // pieces that an operand is read before its use, of four products or dims / 32 of 64 cycles each (eight: no faster)
  typedef Four<XT, FOURS> Piece;
  __shared__ float merged[4 * kRows * (DP + 1)];  // [wave][row][DP + 1]
  __shared__ float merged_m[4][kRows], merged_l[4][kRows];
  const AttentionTile tile = attention_tile(a, blockIdx.x / a.kv_heads, (int)(gridDim.x / (unsigned)a.kv_heads), kRows);
  const int rows = tile.tokens * a.group;
  if (tile.first >= rows) return;
  const int head = blockIdx.x % a.kv_heads, lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), col = lane % 32, half = lane / 32;
  const int row = min(tile.first + col, rows - 1), at = row / a.per_group;
  const int64_t query = (int64_t)head * a.group + (row - at * a.group);
  const int sees = a.causal ? at + 1 : tile.tokens;

  float q[E][4];  // dims 8 e + 4 half + j
  {
    const char* from = static_cast<const char*>(a.q.data) + ((tile.begin + at) * a.q.ld_token + query * a.q.ld_head) * SIZE;
    Piece raw[E];
#pragma unroll
    for (int e = 0; e < E; ++e) raw[e].read(from, 8 * e + 4 * half, a.dim);
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int j = 0; j < 4; ++j) q[e][j] = 8 * e + 4 * half + j < a.dim ? raw[e][j] : 0.f;
  }
  float m = kNoScore, l = 0.f;
  f16v o[F];
#pragma unroll
  for (int f = 0; f < F; ++f)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[f][i] = 0.f;

  const char* k_from = static_cast<const char*>(a.k.data) + (tile.begin * a.k.ld_token + head * a.k.ld_head) * SIZE;
  const char* v_from = static_cast<const char*>(a.v.data) + (tile.begin * a.v.ld_token + head * a.v.ld_head) * SIZE;
  // (a dim that is not there: of keys another one is read and 0 taken, since an infinity would make a NaN of the 0 of q that it meets; of values another one, whose sum
  // is not stored.  A token behind the last one is the last one.)
  Piece k[AHEAD];
  unsigned v[AHEAD][F];
  const char* k_row;
  auto read_keys = [&](int e) { k[e % AHEAD].read(k_row, 8 * e + 4 * half, a.dim); };
  int dims = a.dim - 4 * half;
  auto key = [&](int e, int j) { return 8 * e + (FOURS ? 0 : j) < dims ? k[e % AHEAD][j] : 0.f; };
  auto read_values = [&](int k0, int i) {
    const char* from = v_from + min(k0 + i / 4 * 8 + i % 4 + 4 * half, tile.tokens - 1) * a.v.ld_token * SIZE;
#pragma unroll
    for (int f = 0; f < F; ++f) v[i % AHEAD][f] = Piece::one(from, 32 * f + col < a.dim ? 32 * f + col : 0);
  };
  // a place i of values that some row of the tile does not see: what is not finite of it is taken apart, for it must not reach that row, not even times 0
  auto take_apart = [&](int place, int i, float (&x)[F], const f16v& s) {
    float zero = 0.f;
#pragma unroll
    for (int f = 0; f < F; ++f) zero = fmaf(x[f], 0.f, zero);
    if (!__any(zero != 0.f)) return;
#pragma unroll
    for (int f = 0; f < F; ++f) {
      const bool odd = !(fabsf(x[f]) < INFINITY);
      for (unsigned long long left = __ballot(odd); left; left &= left - 1) {
        const int from = __ffsll((long long)left) - 1;  // the lane that has dim 32 f + from % 32 of its place
        const float bad = __shfl(x[f], from), p = __shfl(s[i], from / 32 * 32 + col);
        const int bad_place = place + 4 * (from / 32), in = from % 32;
        // the lane and register of the row's sum: dim in = 8 (r / 4) + 4 half + r % 4
        const bool own = bad_place < sees && half == in / 4 % 2;
#pragma unroll
        for (int r = 0; r < 16; ++r) o[f][r] = own && r == in / 8 * 4 + in % 4 ? fmaf(p, bad, o[f][r]) : o[f][r];
      }
      x[f] = odd ? 0.f : x[f];
    }
  };
  // 32 keys; ALL: every row sees them.  Ends with the first operands of the next step on their way.
  auto step = [&](int k0, auto all) {
    constexpr bool ALL = decltype(all)::value;
    f16v s;
    asm volatile("" : "+v"(dims));  // (else all comparisons with it are made ahead of the loop, and their results spilled)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
#pragma unroll
      for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(key(e, j), q[e][j], s, 0, 0, 0);
      if (e + AHEAD < E) read_keys(e + AHEAD);
      else read_values(k0, e + AHEAD - E);
      __builtin_amdgcn_sched_barrier(0);
    }
    float high = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = !ALL && k0 + i / 4 * 8 + i % 4 + 4 * half >= sees ? -INFINITY : s[i] * a.scale2;
      high = fmaxf(high, s[i]);
    }
    if (__any(high > m + 8.f)) {
      const float raised = fmaxf(m, fmaxf(high, __shfl_xor(high, 32))), factor = __builtin_amdgcn_exp2f(m - raised);
      m = raised;
      l *= factor;
#pragma unroll
      for (int f = 0; f < F; ++f) o[f] *= factor;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(s[i] - m);
      l += s[i];
    }
    k_row = k_from + min(k0 + 4 * kKeys + col, tile.tokens - 1) * a.k.ld_token * SIZE;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float x[F];
#pragma unroll
      for (int f = 0; f < F; ++f) x[f] = Piece::value(v[i % AHEAD][f]);
      if constexpr (!ALL) take_apart(k0 + i / 4 * 8 + i % 4, i, x, s);
#pragma unroll
      for (int f = 0; f < F; ++f) o[f] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[f], s[i], o[f], 0, 0, 0);
      if (i + AHEAD < 16) read_values(k0, i + AHEAD);
      else read_keys(i + AHEAD - 16);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // keys that any row of the tile sees, and that all see
  const int end = a.causal ? min(tile.first + kRows - 1, rows - 1) / a.per_group + 1 : tile.tokens;
  const int full = a.causal ? tile.first / a.per_group + 1 : tile.tokens;
  k_row = k_from + min(wave * kKeys + col, tile.tokens - 1) * a.k.ld_token * SIZE;
#pragma unroll
  for (int e = 0; e < AHEAD; ++e) read_keys(e);
  int k0 = wave * kKeys;
  for (; k0 + kKeys <= full; k0 += 4 * kKeys) step(k0, std::true_type{});
  for (; k0 < end; k0 += 4 * kKeys) step(k0, std::false_type{});
  l += __shfl_xor(l, 32);
  if (half == 0) merged_m[wave][col] = m, merged_l[wave][col] = l;
  for (int f = 0; f < F; ++f)
    for (int i = 0; i < 16; ++i) merged[(wave * kRows + col) * (DP + 1) + 32 * f + i / 4 * 8 + i % 4 + 4 * half] = o[f][i];
  __syncthreads();
  for (int i = threadIdx.x; i < kRows * DP; i += 256) {
    const int r = i / DP, d = i % DP;
    if (tile.first + r >= rows || d >= a.dim) continue;
    float high = merged_m[0][r], total = 0.f, v = 0.f;
    for (int w = 1; w < 4; ++w) high = fmaxf(high, merged_m[w][r]);
    for (int w = 0; w < 4; ++w) {
      const float factor = __builtin_amdgcn_exp2f(merged_m[w][r] - high);
      total = fmaf(factor, merged_l[w][r], total);
      v = fmaf(factor, merged[(w * kRows + r) * (DP + 1) + d], v);
    }
    const int of = (tile.first + r) / a.per_group;
    w4_store(a.out.type, a.out.data, (tile.begin + of) * a.out.ld_token + ((int64_t)head * a.group + (tile.first + r - of * a.group)) * a.out.ld_head + d,
             total == 0.f ? 0.f : v / total);
  }
}

template <int XT, int DP>
hipError_t launch(const Attention& a, hipStream_t st) {
  const dim3 grid((unsigned)(attention_tiles(a, kRows) * a.kv_heads));
  if (a.dim % 4 == 0) hipLaunchKernelGGL((attention_any_kernel<XT, DP, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((attention_any_kernel<XT, DP, false>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}
template <int XT>
hipError_t of(const Attention& a, hipStream_t st) {
  return a.dim <= 64 ? launch<XT, 64>(a, st) : a.dim <= 96 ? launch<XT, 96>(a, st) : a.dim <= 128 ? launch<XT, 128>(a, st) : launch<XT, 256>(a, st);
}

}  // namespace

hipError_t oz2_attention_any(const Attention& a, hipStream_t st) {
  return a.q.type == OZ2_F32 ? of<OZ2_F32>(a, st) : a.q.type == OZ2_BF16 ? of<OZ2_BF16>(a, st) : of<OZ2_F16>(a, st);
}
