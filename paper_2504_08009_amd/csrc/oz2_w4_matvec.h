// The kernel of oz2_w4_matvec and its launch for one type of x (oz2_w4_f32.hip, oz2_w4_bf16.hip, oz2_w4_f16.hip).
#ifndef OZ2_W4_MATVEC_H
#define OZ2_W4_MATVEC_H

#include "oz2_w4_tile.h"
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

constexpr int kWaves = 8;
constexpr int kLds = 156 * 1024;

// How a launch of tiles cuts the inner dimension: `split` waves share two tiles of sixteen rows, wave s of them takes runs of blocks s, s + split, ... of
// every chunk; x is brought into LDS a chunk of blocks at a time.
struct Cut {
  int split_log, waves, chunk, chunks, pitch, reduce_at;  // waves: of a workgroup
};

template <int XT, int SPB, int RT, bool WIDE, bool ZEROS>
__global__ void __launch_bounds__(64 * kWaves) w4_tile_kernel(W4Rows w, int scale_type, Cut cut, int t, float alpha, const char* x, int64_t ldx, float beta,
                                                              const void* c, int64_t ldc, int y_type, void* y, int64_t ldy) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int split = 1 << cut.split_log, s = wave & (split - 1);
  const int64_t pair = (int64_t)blockIdx.x * (cut.waves >> cut.split_log) + (wave >> cut.split_log);
  const bool in = pair * 32 < w.n;
  const int row[2] = {(int)(in ? pair * 32 : 0), (int)(in ? min(pair * 32 + 16, (int64_t)w.n - 1) : 0)};
  const W4Rows both[2] = {w, w};
  const int first = blockIdx.y * 4 * RT, tokens = min(4 * RT, t - first);
  const char* lane_x = lds + w4_row_of_x<w4_parts<XT>()>(lane % 16, tokens, cut.pitch);
  auto row_of = [&](int token) { return (first + token) * ldx; };
  W4Two<XT, SPB, RT, WIDE, ZEROS> two;
  two.init(both, row, scale_type);
  const int owner = w.full / kW4Run & (split - 1);  // of the block behind the whole ones
  float sum[2][RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) sum[0][r] = sum[1][r] = 0.f;
  // Chunks too are walked from a place of its own for every workgroup.
  int at = cut.chunks > 1 ? blockIdx.x % cut.chunks : 0;
  for (int done = 0; done < cut.chunks; ++done) {
    const int start = at * cut.chunk, end = min(start + cut.chunk, w.full);  // of whole blocks (none: end <= start)
    const bool last = at == cut.chunks - 1, ragged = last && w.full * kW4Block < w.k;
    const int first_run = start / kW4Run + s, runs = (end + kW4Run - 1) / kW4Run;
    typename W4Two<XT, SPB, RT, WIDE, ZEROS>::Ahead ahead;
    const typename W4Two<XT, SPB, RT, WIDE, ZEROS>::Walk walk(first_run, split, (runs - first_run + split - 1) >> cut.split_log, end, (unsigned)pair);
    if (w.full) two.begin(w, walk, ahead);
    if (done) __syncthreads();
    w4_stage<XT>([&](int token) { return x + row_of(token) * (XT == OZ2_F32 ? 4 : 2); }, tokens, w.k, start, end - start + ragged, lds, cut.pitch, 64 * cut.waves);
    __syncthreads();
    if (in) {
      two.multiply(w, walk, start, ahead, lane_x, cut.pitch, sum);
      if (ragged && s == owner) two.multiply_tail(both, row, lane_x + (w.full - start) * kW4Block * 2, cut.pitch, sum);
    }
    at = last ? 0 : at + 1;
  }
  bool again = false;
#pragma unroll
  for (int r = 0; r < 2 * RT; ++r) again |= !(fabsf(sum[r / RT][r % RT]) < INFINITY) && lane / 16 + 4 * (r % RT) < tokens;
  if (in && __ballot(again)) {
    float plain[2][RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) plain[0][r] = plain[1][r] = 0.f;
#pragma unroll 1
    for (int b = 0; b <= w.full; ++b)
      if (b == w.full ? s == owner : (b / kW4Run & (split - 1)) == s)
        two.block_plain(both, row, b, [&](int r, int k) {
          const int token = lane / 16 + 4 * r;
          return token < tokens ? w4_load(XT, x, row_of(token) + k) : 0.f;
        }, plain);
#pragma unroll
    for (int r = 0; r < 2 * RT; ++r)
      if (!(fabsf(sum[r / RT][r % RT]) < INFINITY)) sum[r / RT][r % RT] = plain[r / RT][r % RT];
  }
  if (split > 1) {
    float* part = reinterpret_cast<float*>(lds + cut.reduce_at) + lane;
#pragma unroll
    for (int r = 0; r < 2 * RT; ++r) part[(wave * 2 * RT + r) * 64] = sum[r / RT][r % RT];
    __syncthreads();
    if (s) return;
    for (int i = 1; i < split; ++i)
#pragma unroll
      for (int r = 0; r < 2 * RT; ++r) sum[r / RT][r % RT] += part[((wave + i) * 2 * RT + r) * 64];
  }
#pragma unroll
  for (int i = 0; i < 2 * RT; ++i) {
    const int token = lane / 16 + 4 * (i % RT);
    const int64_t to = pair * 32 + i / RT * 16 + lane % 16;
    if (token >= tokens || to >= w.n) continue;
    float v = alpha * sum[i / RT][i % RT];
    if (beta != 0.f) v = fmaf(beta, w4_load(y_type, c, (first + token) * ldc + to), v);
    w4_store(y_type, y, (first + token) * ldy + to, v);
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
  // Three workgroups a compute unit, each with x in its registers, which walk as many batches as all others.  Three fit with one 16-bit vector and no
  // zero points (76 registers); two with zero points, two 16-bit vectors or one FP32 vector (83 to 111) and one with two FP32 vectors (155 to 159):
  // there the last ones begin when the first are done.
  const int most = oz2_w4_compute_units() * 3, needed = (batches + per - 1) / per, rounds = (needed + most - 1) / most, grid = (needed + rounds - 1) / rounds;
  hipLaunchKernelGGL((w4_vector_kernel<XT, T, ST, ZEROS>), dim3(grid), dim3(64 * kWaves), 0, a.st, a.w, split_log, a.alpha,
                     static_cast<const char*>(a.x), a.ldx, a.beta, a.c, a.ldc, a.y_type, a.y, a.ldy);
  return hipGetLastError();
}

template <int XT, int SPB, int RT, bool WIDE, bool ZEROS>
hipError_t launch_tile(const W4Call& a) {
  constexpr int P = w4_parts<XT>();
  const int tokens = a.t < 4 * RT ? a.t : 4 * RT;
  const int64_t pairs = (a.w.n + 31) / 32;
  const int blocks = (a.w.k + kW4Block - 1) / kW4Block;
  const int cus = oz2_w4_compute_units();
  Cut cut;
  cut.split_log = 0;
  while (cut.split_log < 3 && (pairs << cut.split_log) < 8 * cus && (kW4Run << cut.split_log) < blocks) ++cut.split_log;
  auto lay = [&](int chunk) {
    cut.chunk = chunk;
    cut.pitch = chunk * kW4Block * 2 + 16;
    cut.reduce_at = tokens * P * cut.pitch;
    return cut.reduce_at + (cut.split_log ? kWaves * 2 * RT * 64 * 4 : 0);
  };
  int lds = lay(blocks);
  if (lds > kLds) {  // not in one piece: as many runs for each wave of a pair as fit, fewer waves a pair where that is none
    while (cut.split_log && lay(kW4Run << cut.split_log) > kLds) --cut.split_log;
    int each = 1;
    while (lay((each + 1) * kW4Run << cut.split_log) <= kLds) ++each;
    lds = lay(each * kW4Run << cut.split_log);
  }
  cut.chunks = (blocks + cut.chunk - 1) / cut.chunk;
  // pairs of tiles that a workgroup takes: as many as still leave every compute unit one
  int per = 1;
  while ((per * 2 << cut.split_log) <= kWaves && pairs >= 2 * per * cus) per *= 2;
  cut.waves = per << cut.split_log;
  static const hipError_t set = hipFuncSetAttribute(reinterpret_cast<const void*>(&w4_tile_kernel<XT, SPB, RT, WIDE, ZEROS>),
                                                    hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
  if (set != hipSuccess) return set;
  hipLaunchKernelGGL((w4_tile_kernel<XT, SPB, RT, WIDE, ZEROS>), dim3((unsigned)((pairs + per - 1) / per), (unsigned)((a.t + 4 * RT - 1) / (4 * RT))),
                     dim3(64 * cut.waves), lds, a.st, a.w, a.scale_type, cut, a.t, a.alpha, static_cast<const char*>(a.x), a.ldx, a.beta, a.c, a.ldc, a.y_type,
                     a.y, a.ldy);
  return hipGetLastError();
}

template <int XT, int SPB, int RT>
hipError_t launch_scales(const W4Call& a) {
  if (a.scale_type == OZ2_F32) return a.w.zeros ? launch_tile<XT, SPB, RT, true, true>(a) : launch_tile<XT, SPB, RT, true, false>(a);
  return a.w.zeros ? launch_tile<XT, SPB, RT, false, true>(a) : launch_tile<XT, SPB, RT, false, false>(a);
}
template <int XT, int SPB>
hipError_t launch_tokens(const W4Call& a) {
  return a.t <= 4 ? launch_scales<XT, SPB, 1>(a) : launch_scales<XT, SPB, 4>(a);
}

template <int XT, int T, bool ZEROS>
hipError_t launch_rows(const W4Call& a) {
  return a.scale_type == OZ2_F32    ? launch_vector<XT, T, OZ2_F32, ZEROS>(a)
         : a.scale_type == OZ2_BF16 ? launch_vector<XT, T, OZ2_BF16, ZEROS>(a)
                                    : launch_vector<XT, T, OZ2_F16, ZEROS>(a);
}
template <int XT, int T>
hipError_t launch_rows(const W4Call& a) {
  return a.w.zeros ? launch_rows<XT, T, true>(a) : launch_rows<XT, T, false>(a);
}

}  // namespace

template <int XT>
hipError_t oz2_w4_matvec_of(const W4Call& a, int64_t group) {
  if (a.t <= 2 && a.w.k >= 1024 && a.w.k <= kW4Span * kWaves) return a.t == 1 ? launch_rows<XT, 1>(a) : launch_rows<XT, 2>(a);
  return group == 32 ? launch_tokens<XT, 4>(a) : group == 64 ? launch_tokens<XT, 2>(a) : launch_tokens<XT, 1>(a);
}
#endif
#endif
