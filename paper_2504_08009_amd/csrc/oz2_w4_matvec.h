// The kernel of oz2_w4_matvec and its launch for one type of x (oz2_w4_f32.hip, oz2_w4_bf16.hip, oz2_w4_f16.hip).
#ifndef OZ2_W4_MATVEC_H
#define OZ2_W4_MATVEC_H

#include "oz2_w4_vector.h"

struct W4Call {
  W4Rows w;
  int scale_type;
  int t;
  float alpha, beta;
  const void *x, *c;
  int64_t ldx, ldc, ldy;
  int y_type;
  void* y;
  hipStream_t st;
};
template <int XT>
hipError_t oz2_w4_matvec_of(const W4Call& a, int64_t group);
int oz2_w4_compute_units();

#ifdef __HIPCC__
namespace {

#ifndef W4_WANT
#define W4_WANT 2048
#endif
constexpr int kWaves = 8;
constexpr int kLds = 64 * 1024;

// How a launch cuts the inner dimension: `split` waves share a tile of sixteen rows, wave s of them takes blocks s, s + split, ... of every chunk;
// x is brought into LDS a chunk of blocks at a time.
struct Cut {
  int split_log, chunk, chunks, pitch, sums_at, flags_at, reduce_at;
};

template <int XT, int SPB, int RT, int ST, bool ZEROS>
__global__ void __launch_bounds__(64 * kWaves) w4_matvec_kernel(W4Rows w, Cut cut, int t, float alpha, const void* x, int64_t ldx, float beta,
                                                                const void* c, int64_t ldc, int y_type, void* y, int64_t ldy) {
#ifndef W4_U
#define W4_U 4
#endif
  constexpr int U = W4_U;  // blocks of a wave in flight
  constexpr int PIECES = RT == 1 ? 2 : 4;  // pieces of x of a thread in flight
  extern __shared__ char lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int split = 1 << cut.split_log, s = wave & (split - 1);
  const int64_t tile = (int64_t)blockIdx.x * (kWaves >> cut.split_log) + (wave >> cut.split_log);
  const int64_t row = tile * 16 + lane % 16;
  const int first = blockIdx.y * 4 * RT, tokens = min(4 * RT, t - first);
  const W4Lane l = w4_lane<ST>(w, row);
  float* sums = reinterpret_cast<float*>(lds + cut.sums_at);
  unsigned* flags = reinterpret_cast<unsigned*>(lds + cut.flags_at);
  const char* lane_x = lds + min(w4_token<RT>(lane % 16), tokens - 1) * w4_parts<XT>() * cut.pitch;
  auto row_of = [&](int token) { return (first + token) * ldx; };
  const bool in = tile * 16 < w.n;
  float sum[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) sum[r] = 0.f;

  // Chunks, and blocks inside one, are walked from a place of its own for every workgroup and tile: rows lie whole pages apart as a rule, and
  // where all waves stand at the same inner index, they ask the same few memory channels.
  int at = cut.chunks > 1 ? blockIdx.x % cut.chunks : 0;
  for (int done = 0; done < cut.chunks; ++done) {
    const int start = at * cut.chunk, whole = min(cut.chunk, w.full - start);  // (whole blocks: 0 or more)
    const bool last = at == cut.chunks - 1, ragged = last && w.full * kW4Block < w.k;
    const int count = in ? (whole - s + split - 1) >> cut.split_log : 0;  // whole blocks of this wave
    const int turn = count > 1 ? (int)((unsigned)tile * 4 % (unsigned)count) : 0;
    auto block = [&](int i) {
      i = min(i, count - 1) + turn;
      return start + s + ((i < count ? i : i - count) << cut.split_log);
    };
    const W4Stage stage = {static_cast<const char*>(x), (int64_t)start * kW4Block, tokens, w.k, (whole + ragged) * (kW4Block / 8)};
    const int pieces = tokens * stage.eights;
    W4Regs<SPB, ST> regs[U];
    W4Tail<SPB> tail;
    if (count)
      w4_each<U>([&](auto u) __attribute__((always_inline)) { regs[u.value] = w4_fetch<SPB, ST, ZEROS>(w, l, block(u.value)); });
    const bool tail_here = ragged && in && (whole & (split - 1)) == s;
    if (tail_here) tail = w4_fetch_tail<SPB, ST, ZEROS>(w, l);
    if (done) __syncthreads();
    bool plain = false;
#pragma unroll 1
    for (int piece = threadIdx.x; piece < pieces; piece += PIECES * 64 * kWaves) {
      W4Raw<XT> raw[PIECES];
      w4_each<PIECES>([&](auto i) __attribute__((always_inline)) {
        raw[i.value] = w4_stage_load<XT>(stage, row_of, min(piece + i.value * 64 * kWaves, pieces - 1));
      });
      w4_each<PIECES>([&](auto i) __attribute__((always_inline)) {
        if (piece + i.value * 64 * kWaves < pieces)
          plain |= w4_stage_store<XT, SPB, RT>(stage, raw[i.value], piece + i.value * 64 * kWaves, lds, cut.pitch, sums);
      });
    }
    const bool any = __ballot(plain) != 0;
    if (lane == 0) flags[wave] = any;
    __syncthreads();
    unsigned seen = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) seen |= flags[i];
    if (__builtin_amdgcn_readfirstlane(seen)) {
#pragma unroll 1
      for (int i = 0; i < count + tail_here; ++i)
        w4_block_plain<SPB, ST, RT>(w, l, ZEROS, i < count ? block(i) : w.full, [&](int r, int k) {
          const int token = lane / 16 + 4 * r;
          return token < tokens ? w4_load(XT, x, row_of(token) + k) : 0.f;
        }, sum);
    } else {
#pragma unroll 1
      for (int i = 0; i < count; i += U)
        w4_each<U>([&](auto u) __attribute__((always_inline)) {
          const int b = block(i + u.value) - start;
          if (i + u.value < count)
            w4_whole<XT, SPB, ST, ZEROS, RT>(regs[u.value], lane_x + b * kW4Block * 2, cut.pitch, sums + b * SPB * 4 * RT, sum);
          regs[u.value] = w4_fetch<SPB, ST, ZEROS>(w, l, block(i + u.value + U));
        });
      if (tail_here) {
        const int b = w.full - start;
        w4_tail<XT, SPB, ST, RT>(w, tail, lane_x + b * kW4Block * 2, cut.pitch, sums + b * SPB * 4 * RT, sum);
      }
    }
    at = last ? 0 : at + 1;
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
    float v = cut.chunks ? alpha * sum[r] : 0.f;
    if (beta != 0.f) v = fmaf(beta, w4_load(y_type, c, (first + token) * ldc + row), v);
    w4_store(y_type, y, (first + token) * ldy + row, v);
  }
}

// One or two vectors: four rows at a time for each `1 << split_log` waves, which share their inner dimension (a span of 2048 each).
constexpr int kRounds = 8;  // between two barriers

template <int XT, int T, int ST, bool ZEROS>
__global__ void __launch_bounds__(64 * kWaves) w4_vector_kernel(W4Rows w, int split_log, float alpha, const char* x, int64_t ldx, float beta, const void* c,
                                                                int64_t ldc, int y_type, void* y, int64_t ldy) {
  __shared__ float part[2][kRounds][kWaves][4][T];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int split = 1 << split_log, s = wave & (split - 1), per = kWaves >> split_log;
  const int batches = (w.n + 3) / 4, step = gridDim.x * per, first = blockIdx.x * per;
  const int unit = s * 64 + lane;
  const W4Place at = w4_place(w, unit);
  const bool ragged = __ballot(at.cut != 0) != 0;
  W4Rows4<XT, T, ST, ZEROS, 1> rows;
  int b = first + (wave >> split_log);
  auto row_of = [&](int batch) { return [&, batch](int i) { return w4_row<ST, 1>(w, batch * 4, i); }; };
  auto vector = [&](int t) { return x + t * ldx * (XT == OZ2_F32 ? 4 : 2); };
  rows.fetch(row_of(b), at);
  W4X<XT> kept[T];
  const unsigned plain = w4_take_x<XT, T>(w.k, unit, vector, kept);
  auto finish = [&](int64_t row, int t, float v) {
    float u = alpha * v;
    if (beta != 0.f) u = fmaf(beta, w4_load(y_type, c, t * ldc + row), u);
    w4_store(y_type, y, t * ldy + row, u);
  };
  const int rounds = (batches - first + step - 1) / step;  // of the workgroup: its first wave has the most
  for (int i = 0; i < rounds; ++i, b += step) {
    float sum[4][T];
    rows.multiply(at, kept, ragged, sum);
    if (plain) rows.multiply_plain(plain, w.k, w.group, row_of(b), vector, unit, sum);
    if (i + 1 < rounds) rows.fetch(row_of(b + step), at);
    float v[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      float one[1];
      w4_sum4<1>(sum[0][t], sum[1][t], sum[2][t], sum[3][t], one);
      v[t] = one[0];
    }
    const int t = lane % 16;
    if (split == 1) {
      const int64_t row = (int64_t)b * 4 + lane / 16;
      if (t < T && row < w.n) finish(row, t, T == 2 && t ? v[T - 1] : v[0]);
      continue;
    }
    if (t < T) part[i / kRounds % 2][i % kRounds][wave][lane / 16][t] = T == 2 && t ? v[T - 1] : v[0];
    if (i % kRounds != kRounds - 1 && i + 1 < rounds) continue;
    __syncthreads();
    const int since = i / kRounds * kRounds;  // rounds since .. i have been left in `part`: (row, vector) for (row, vector) to a thread
    for (int j = threadIdx.x; j < (i + 1 - since) * per * 4 * T; j += 64 * kWaves) {
      const int tj = j % T, r = j / T % 4, group = j / (4 * T) % per, round = j / (4 * T) / per;
      float u = 0.f;
      for (int q = 0; q < split; ++q) u += part[i / kRounds % 2][round][group * split + q][r][tj];
      const int64_t row = ((int64_t)(since + round) * step + first + group) * 4 + r;
      if (row < w.n) finish(row, tj, u);
    }
  }
}

template <int XT, int T, int ST, bool ZEROS>
hipError_t launch_vector(const W4Call& a) {
  int split_log = 0;
  while ((kW4Span << split_log) < a.w.k) ++split_log;
  const int per = kWaves >> split_log, batches = (a.w.n + 3) / 4;
  // three workgroups a compute unit fit; each has x in its registers and walks as many batches as all others
  const int most = oz2_w4_compute_units() * 3, needed = (batches + per - 1) / per, rounds = (needed + most - 1) / most, grid = (needed + rounds - 1) / rounds;
  hipLaunchKernelGGL((w4_vector_kernel<XT, T, ST, ZEROS>), dim3(grid), dim3(64 * kWaves), 0, a.st, a.w, split_log, a.alpha,
                     static_cast<const char*>(a.x), a.ldx, a.beta, a.c, a.ldc, a.y_type, a.y, a.ldy);
  return hipGetLastError();
}

template <int XT, int SPB, int RT, int ST, bool ZEROS>
hipError_t launch(const W4Call& a) {
  constexpr int P = w4_parts<XT>();
  const int tokens = a.t < 4 * RT ? a.t : 4 * RT;
  const int64_t tiles = (a.w.n + 15) / 16;
  const int blocks = (int)((a.w.k + (int64_t)kW4Block - 1) / kW4Block);
  Cut cut;
  cut.split_log = 0;
  while (cut.split_log < 3 && (tiles << cut.split_log) < W4_WANT && (2 << cut.split_log) <= blocks) ++cut.split_log;
  auto lay = [&](int chunk) {
    cut.chunk = chunk;
    cut.pitch = chunk * kW4Block * 2 + 16;
    cut.sums_at = tokens * P * cut.pitch;
    cut.flags_at = cut.sums_at + chunk * SPB * 4 * RT * 4;
    cut.reduce_at = cut.flags_at + kWaves * 4;
    return cut.reduce_at + (cut.split_log ? kWaves * RT * 64 * 4 : 0);
  };
  int lds = lay(blocks > 0 ? blocks : 1);
  if (lds > kLds) {  // not in one piece: as many blocks for each wave of a tile as fit, fewer waves a tile where that is none
    while (lay(1 << cut.split_log) > kLds) --cut.split_log;
    int each = 1;
    while (lay((each + 1) << cut.split_log) <= kLds) ++each;
    lds = lay(each << cut.split_log);
  }
  cut.chunks = (blocks + cut.chunk - 1) / cut.chunk;
  const int per = kWaves >> cut.split_log;
  hipLaunchKernelGGL((w4_matvec_kernel<XT, SPB, RT, ST, ZEROS>), dim3((unsigned)((tiles + per - 1) / per), (unsigned)((a.t + 4 * RT - 1) / (4 * RT))),
                     dim3(64 * kWaves), lds, a.st, a.w, cut, a.t, a.alpha, a.x, a.ldx, a.beta, a.c, a.ldc, a.y_type, a.y, a.ldy);
  return hipGetLastError();
}

// f(type of the scales, whether there are zero points), as constants
template <class F>
hipError_t by_scales(const W4Call& a, F f) {
  auto zeros = [&](auto st) { return a.w.zeros ? f(st, W4Index<1>{}) : f(st, W4Index<0>{}); };
  return a.scale_type == OZ2_F32 ? zeros(W4Index<OZ2_F32>{}) : a.scale_type == OZ2_BF16 ? zeros(W4Index<OZ2_BF16>{}) : zeros(W4Index<OZ2_F16>{});
}
template <int XT, int SPB, int RT>
hipError_t launch_tile(const W4Call& a) {
  return by_scales(a, [&](auto st, auto zeros) { return launch<XT, SPB, RT, decltype(st)::value, decltype(zeros)::value>(a); });
}
template <int XT, int SPB>
hipError_t launch_tokens(const W4Call& a) {
  return a.t <= 4 ? launch_tile<XT, SPB, 1>(a) : launch_tile<XT, SPB, 4>(a);
}
template <int XT, int T>
hipError_t launch_rows(const W4Call& a) {
  return by_scales(a, [&](auto st, auto zeros) { return launch_vector<XT, T, decltype(st)::value, decltype(zeros)::value>(a); });
}

}  // namespace

template <int XT>
hipError_t oz2_w4_matvec_of(const W4Call& a, int64_t group) {
  if (a.t <= 2 && a.w.k >= 1024 && a.w.k <= kW4Span * kWaves) return a.t == 1 ? launch_rows<XT, 1>(a) : launch_rows<XT, 2>(a);
  return group == 32 ? launch_tokens<XT, 4>(a) : group == 64 ? launch_tokens<XT, 2>(a) : launch_tokens<XT, 1>(a);
}
#endif
#endif
