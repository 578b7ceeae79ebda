// Products of a matrix held in 4 bits and a few vectors (oz2_w4_matvec).
#include "oz2_w4_core.h"

namespace {

constexpr int kWaves = 8;
constexpr int kLds = 64 * 1024;

// How a launch cuts the inner dimension: `split` waves share a tile of sixteen rows, wave s of them takes blocks s, s + split, ...; x is brought
// into LDS `chunk` blocks at a time.
struct Cut {
  int split_log, chunk, pitch, sums_at, flags_at, reduce_at;
};

template <int XT, int SPB, int RT>
__global__ void __launch_bounds__(64 * kWaves) w4_matvec_kernel(W4Rows w, Cut cut, int t, float alpha, const void* x, int64_t ldx, float beta,
                                                                const void* c, int64_t ldc, int y_type, void* y, int64_t ldy) {
  constexpr int U = RT == 4 ? 2 : 4;  // blocks of a wave in flight
  extern __shared__ char lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int split = 1 << cut.split_log, s = wave & (split - 1);
  const int64_t tile = (int64_t)blockIdx.x * (kWaves >> cut.split_log) + (wave >> cut.split_log);
  const int64_t row = tile * 16 + lane % 16;
  const int first = blockIdx.y * 4 * RT, tokens = min(4 * RT, t - first);
  const W4Lane l = w4_lane(w, row);
  float* sums = reinterpret_cast<float*>(lds + cut.sums_at);
  unsigned* flags = reinterpret_cast<unsigned*>(lds + cut.flags_at);
  const int mine = tile * 16 < w.n ? (w.blocks - s + split - 1) >> cut.split_log : 0;  // blocks of this wave

  W4Regs<SPB> regs[U];
  w4_each<U>([&](auto u) __attribute__((always_inline)) {
    if (u.value < mine) regs[u.value] = w4_fetch<SPB>(w, l, s + (u.value << cut.split_log));
  });

  float sum[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) sum[r] = 0.f;
  const char* lane_x = lds + min(w4_token<RT>(lane % 16), tokens - 1) * w4_parts<XT>() * cut.pitch;
  auto row_of = [&](int token) { return (first + token) * ldx; };
  for (int start = 0; start < w.blocks; start += cut.chunk) {
    const int length = min(cut.chunk, w.blocks - start);
    if (start) __syncthreads();
    const bool plain = w4_stage<XT, SPB, RT>(x, row_of, tokens, w.k, start * kW4Block, length * kW4Block, lds, cut.pitch, sums, 64 * kWaves);
    const bool any = __ballot(plain) != 0;
    if (lane == 0) flags[wave] = any;
    __syncthreads();
    unsigned seen = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) seen |= flags[i];
    const bool slow = __builtin_amdgcn_readfirstlane(seen) != 0;
    const int end = start + cut.chunk < w.blocks ? min(mine, (start + cut.chunk) >> cut.split_log) : mine;
    if (slow) {
#pragma unroll 1
      for (int i = start >> cut.split_log; i < end; ++i)
        w4_block_plain<SPB, RT>(w, l, s + (i << cut.split_log), [&](int r, int k) {
          const int token = lane / 16 + 4 * r;
          return token < tokens ? w4_load(XT, x, row_of(token) + k) : 0.f;
        }, sum);
      w4_each<U>([&](auto u) __attribute__((always_inline)) {
        if (end + u.value < mine) regs[u.value] = w4_fetch<SPB>(w, l, s + ((end + u.value) << cut.split_log));
      });
      continue;
    }
#pragma unroll 1
    for (int i = start >> cut.split_log; i < end; i += U)
      w4_each<U>([&](auto u) __attribute__((always_inline)) {
        if (i + u.value < end) {
          const int at = s + ((i + u.value) << cut.split_log) - start;
          w4_block<XT, SPB, RT>(w, regs[u.value], lane_x + at * kW4Block * 2, cut.pitch, sums + at * SPB * 4 * RT, sum);
        }
        if (i + u.value + U < mine) regs[u.value] = w4_fetch<SPB>(w, l, s + ((i + u.value + U) << cut.split_log));
      });
  }
  if (split > 1) {
    float* part = reinterpret_cast<float*>(lds + cut.reduce_at) + lane;
#pragma unroll
    for (int r = 0; r < RT; ++r) part[(wave * RT + r) * 64] = sum[r];
    __syncthreads();
    if (s) return;
    for (int i = 1; i < split; ++i)
#pragma unroll
      for (int r = 0; r < RT; ++r) sum[r] += part[((wave + i) * RT + r) * 64];
  }
  if (row >= w.n) return;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int token = lane / 16 + 4 * r;
    if (token >= tokens) continue;
    float v = w.blocks ? alpha * sum[r] : 0.f;
    if (beta != 0.f) v = fmaf(beta, w4_load(y_type, c, (first + token) * ldc + row), v);
    w4_store(y_type, y, (first + token) * ldy + row, v);
  }
}

struct Call {
  W4Rows w;
  int t;
  float alpha, beta;
  const void *x, *c;
  int64_t ldx, ldc, ldy;
  int y_type;
  void* y;
  hipStream_t st;
};

template <int XT, int SPB, int RT>
hipError_t launch(const Call& a) {
  constexpr int U = RT == 4 ? 2 : 4, P = w4_parts<XT>();
  const int tokens = a.t < 4 * RT ? a.t : 4 * RT;
  const int64_t tiles = (a.w.n + 15) / 16;
  Cut cut;
  cut.split_log = 0;
  while (cut.split_log < 3 && (tiles << cut.split_log) < 2048 && (2 << cut.split_log) <= a.w.blocks) ++cut.split_log;
  auto lay = [&](int chunk) {
    cut.chunk = chunk;
    cut.pitch = chunk * kW4Block * 2 + 16;
    cut.sums_at = tokens * P * cut.pitch;
    cut.flags_at = cut.sums_at + chunk * SPB * 4 * RT * 4;
    cut.reduce_at = cut.flags_at + kWaves * 4;
    return cut.reduce_at + (cut.split_log ? kWaves * RT * 64 * 4 : 0);
  };
  int step = U << cut.split_log, lds;
  if ((lds = lay(a.w.blocks)) > kLds) {  // not in one piece: the most steps that fit, fewer waves a tile where not even one does
    while (lay(step) > kLds) --cut.split_log, step /= 2;
    int steps = 1;
    while (lay((steps + 1) * step) <= kLds) ++steps;
    lds = lay(steps * step);
  }
  const int per = kWaves >> cut.split_log;
  hipLaunchKernelGGL((w4_matvec_kernel<XT, SPB, RT>), dim3((unsigned)((tiles + per - 1) / per), (unsigned)((a.t + 4 * RT - 1) / (4 * RT))), dim3(64 * kWaves),
                     lds, a.st, a.w, cut, a.t, a.alpha, a.x, a.ldx, a.beta, a.c, a.ldc, a.y_type, a.y, a.ldy);
  return hipGetLastError();
}

template <int XT, int SPB>
hipError_t launch_tokens(const Call& a) {
  return a.t <= 4 ? launch<XT, SPB, 1>(a) : a.t <= 8 ? launch<XT, SPB, 2>(a) : launch<XT, SPB, 4>(a);
}
template <int XT>
hipError_t launch_group(const Call& a, int64_t group) {
  return group == 32 ? launch_tokens<XT, 4>(a) : group == 64 ? launch_tokens<XT, 2>(a) : launch_tokens<XT, 1>(a);
}

}  // namespace

W4Rows oz2_w4_rows(const oz2_w4_matrix& m) {
  W4Rows w;
  w.codes = static_cast<const uint8_t*>(m.codes);
  w.scales = static_cast<const char*>(m.scales);
  w.zeros = static_cast<const uint8_t*>(m.zeros);
  w.ld_codes = m.ld_codes, w.ld_scales = m.ld_scales, w.ld_zeros = m.ld_zeros;
  w.n = (int)m.n, w.k = (int)m.k;
  w.bytes = (w.k + 1) / 2;
  w.blocks = (w.k + kW4Block - 1) / kW4Block;
  w.groups = (int)((m.k + m.group - 1) / m.group);
  w.per_group = m.group <= kW4Block ? 1 : m.group / kW4Block < w.blocks ? (int)(m.group / kW4Block) : w.blocks > 1 ? w.blocks : 1;
  w.shift = (w.per_group & (w.per_group - 1)) == 0 ? __builtin_ctz(w.per_group) : -1;
  w.scale_type = m.scale_type;
  return w;
}

hipError_t oz2_launch_w4_matvec(const oz2_w4_matrix& m, int64_t t, float alpha, int x_type, const void* x, int64_t ldx, float beta,
                                const void* c, int64_t ldc, int y_type, void* y, int64_t ldy, hipStream_t st) {
  const Call a = {oz2_w4_rows(m), (int)t, alpha, beta, x, c, ldx, ldc, ldy, y_type, y, st};
  return x_type == OZ2_F32 ? launch_group<OZ2_F32>(a, m.group) : x_type == OZ2_BF16 ? launch_group<OZ2_BF16>(a, m.group) : launch_group<OZ2_F16>(a, m.group);
}
