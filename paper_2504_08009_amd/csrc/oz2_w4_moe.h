// A layer of gated experts held in 4 bits (oz2_w4_moe): what its kernels share.  Dispatch in oz2_w4_moe.hip, the products with the
// experts by type of the tokens in oz2_w4_moe_f32.hip, oz2_w4_moe_bf16.hip, oz2_w4_moe_f16.hip, the second ones in oz2_w4_moe_down.hip.
//
// Three launches (router; choice, gate and up; down with the sum over a token's experts) where an expert has a token at the most as a rule, four (the
// sum in its own) where several share its weights, which are then read once for up to sixteen.  One token through 8 of 128 experts of
// 2048 x 1024: 20.8 us = 3.8 + 11 + 6 for 26 MB, each launch at its own latency; 4 tokens, 6 of 64 of 4096 x 1024: 56 us = 6 + 29 + 20
// for 140 MB; 16, 6 of 64 of 2048 x 1408: 86 us = 5 + 45 + 35 + 4 for 210 MB.
#ifndef OZ2_W4_MOE_H
#define OZ2_W4_MOE_H

#include "oz2_w4_tile.h"
#include "oz2_w4_vector.h"

constexpr int kMoeTokens = 32;                               // of a sequence of launches; more tokens take several
constexpr int kMoePlaces = kMoeTokens * OZ2_MOE_MAX_TOP_K;   // a token's j-th expert: place token * top_k + j

// One call, for at most kMoeTokens of its tokens.
struct MoeCall {
  int t, d, f, experts, top_k;
  int score, renormalize, activation;
  float factor;
  const float* bias;
  const uint8_t* active;
  const char* x;
  int64_t ldx;
  W4Rows gate, up, down;                                     // matrix 0 of the stacks
  int64_t code_strides[3], scale_strides[3], zero_strides[3];  // (scales: in bytes)
  int y_type;
  char* y;
  int64_t ldy;
  float* logits;    // experts x t
  int* ids;         // top_k x t
  float* weights;
  float* h;         // f x places
  float* part;      // d x places: products of the down matrices times the weights
  int* chosen;      // of the layer's experts: number that somebody chose, then each with its first entry in `list`, then the places by expert
  int tiles;        // vectors of an expert at a time: 1, by the vector units, or 4 or 16, by the matrix cores
  int direct;       // the second products of a token's places are summed where they are formed
  hipStream_t st;
};

W4Rows oz2_w4_rows(const oz2_w4_matrix& m);
template <int XT>
hipError_t oz2_moe_gate_up(const MoeCall& c, const oz2_w4_matrix& gate);
hipError_t oz2_moe_down(const MoeCall& c, const oz2_w4_matrix& down);
int oz2_w4_compute_units();

#ifdef __HIPCC__
namespace {

constexpr int kMoeWaves = 4, kMoeRounds = 8;
constexpr int kMoeLongest = kMoeWaves * kW4Span;  // inner dimension

// Places by the expert that they chose.
struct Chosen {
  int count;                             // experts that somebody chose
  short expert[kMoePlaces];              // in ascending order
  short first[kMoePlaces + 1];           // where the places of the i-th begin
  short place[kMoePlaces];
};

// How the experts' batches (or groups of rows) are dealt out: items of up to kMoeRounds neighbouring ones, neighbouring items to neighbouring workgroups,
// which then read neighbouring memory (where each has an even share of its own, all read a fixed distance apart, and 32
// tokens through 8 of 128 experts of 4096 x 2048 took 864 in the place of 632 us, both by the vector units).  The size of an item is that with which the busiest
// workgroup has the least to do, `cost` batches beside its own for an item.
struct Items {
  int rounds, of_expert, all;
  __device__ __forceinline__ Items(int experts, int batches, int cost) {
    int least = 0x7FFFFFFF;
    rounds = of_expert = all = 0;
    for (int r = 1; r <= kMoeRounds; ++r) {
      const int n = (batches + r - 1) / r, load = (experts * n + (int)gridDim.x - 1) / (int)gridDim.x * (r + cost);
      if (load < least) least = load, rounds = r, of_expert = n;
    }
    all = experts * of_expert;
  }
};

__device__ __forceinline__ W4Rows w4_of_stack(W4Rows w, int64_t e, int64_t codes, int64_t scales, int64_t zeros) {
  w.codes += e * codes, w.scales += e * scales, w.zeros += e * zeros;
  return w;
}

// Rows of experts times the places that chose them.  A batch is four loads of rows for each `1 << split_log` waves, `loads` of which (4, or 2 beside 2 of a second matrix) are of one matrix.
// row(expert's matrices, row, i): the i-th load of the batch from that row; x(place): vector; out(place, row, sums): called by one
// thread with the sums of the batch's 4 FOLD rows.
template <int XT, int ST, bool ZEROS, int FOLD, class Matrix, class Row, class X, class Out>
__device__ __forceinline__ void moe_products(const Chosen& chosen, int k, int rows, int loads, int split_log, const W4Rows& shape,
                                             float (*part)[kMoeRounds][kMoeWaves][4 * FOLD], Matrix matrix, Row row_of, X vector, Out out) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int split = 1 << split_log, s = wave & (split - 1), group = wave >> split_log, per = kMoeWaves >> split_log;
  const int unit = FOLD == 2 ? lane % 32 : s * 64 + lane, rows_of_batch = loads * FOLD;
  const W4Place at = w4_place(shape, unit);
  const bool ragged = __ballot(at.cut != 0) != 0;
  auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int count = uniform(chosen.count);
  const int batches = (rows + rows_of_batch * per - 1) / (rows_of_batch * per);  // of an expert
  int flip = 0;
  const Items items(count, batches, 2);
  for (int item = blockIdx.x; item < items.all; item += gridDim.x) {  // (an expert's second and later places find the codes in the caches)
    const int a = item / items.of_expert, b = (item - a * items.of_expert) * items.rounds, turns = min(items.rounds, batches - b);
    const int first = uniform(chosen.first[a]), places = uniform(chosen.first[a + 1]) - first;
    const auto m = matrix((int64_t)uniform(chosen.expert[a]));
    auto rows_at = [&](int i) {
      const int row = ((b + i) * per + group) * rows_of_batch;
      return [&, row](int j) { return row_of(m, row, j); };
    };
    for (int p = 0; p < places; ++p) {
      auto x_at = [&](int) { return vector(uniform(chosen.place[first + p])); };
      W4Rows4<XT, 1, ST, ZEROS, FOLD> r;
      r.fetch(rows_at(0), at);
      W4X<XT> kept[1];
      const unsigned plain = w4_take_x<XT, 1>(k, unit, x_at, kept);
      for (int i = 0; i < turns; ++i) {
        float sum[4][1];
        r.multiply(at, kept, ragged, sum);
        if (plain) r.multiply_plain(plain, k, shape.group, rows_at(i), x_at, unit, sum);
        if (i + 1 < turns) r.fetch(rows_at(i + 1), at);
        float v[FOLD];
        w4_sum4<FOLD>(sum[0][0], sum[1][0], sum[2][0], sum[3][0], v);
        if (lane % 16 == 0)
#pragma unroll
          for (int j = 0; j < FOLD; ++j) part[flip][i][wave][w4_row_of_lane<FOLD>(j)] = v[j];
      }
      __syncthreads();
      for (int j = threadIdx.x; j < turns * per; j += 64 * kMoeWaves) {
        const int g = j % per, i = j / per;
        float v[4 * FOLD];
#pragma unroll
        for (int n = 0; n < 4 * FOLD; ++n) v[n] = part[flip][i][g * split][n];
        for (int q = 1; q < split; ++q)
#pragma unroll
          for (int n = 0; n < 4 * FOLD; ++n) v[n] += part[flip][i][g * split + q][n];
        out(chosen.place[first + p], ((b + i) * per + g) * rows_of_batch, v);
      }
      flip ^= 1;
    }
  }
}

// The same on the matrix cores: a wave takes two tiles of sixteen rows, of one matrix or of two, for up to 4 RT places at a time, a workgroup
// rows_of_wave rows for each of its waves.  tile(expert's matrices, t): the matrix of tile t; row(first, t): its first row; out(place, row, sum0,
// sum1): called by the lane that has the sums of row `row` of either tile.
// Three workgroups fit a compute unit by their registers, and x of each, so that they fit by LDS too (two: 16 tokens through 6 of 64 experts of
// 2048 x 1408 take 104 in the place of 86 us; four of them, with up to 4 vectors, 91).  It holds a run of blocks at least.
constexpr int kMoeFit = 3, kMoeLds = 44 * 1024;
template <int XT, int RT>
constexpr int moe_most() { return RT == 4 && w4_parts<XT>() == 3 ? 12 : 4 * RT; }  // places at a time
static_assert(kMoeLds >= 12 * 3 * (kW4Run * kW4Block * 2 + 16) && kMoeLds >= 16 * (kW4Run * kW4Block * 2 + 16), "a run");

template <int XT, int SPB, int RT, bool WIDE, bool ZEROS, class Matrix, class Tile, class First, class X, class Out>
__device__ __forceinline__ void moe_tiles(const Chosen& chosen, int tokens_of_call, int k, int rows, int rows_of_wave, int scale_type, char* lds, Matrix matrix, Tile tile,
                                          First first_row, X vector, Out out) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int count = uniform(chosen.count), blocks = (k + kW4Block - 1) / kW4Block, full = k / kW4Block;
  const int groups = (rows + rows_of_wave * kMoeWaves - 1) / (rows_of_wave * kMoeWaves);
  W4Two<XT, SPB, RT, WIDE, ZEROS> two;
  // Whether x is one piece for every lot that a call of this size can have (a token has an expert once).  Where it is not, the chunks differ with the
  // lot, which follows from what the other tokens have chosen, and the runs are taken in ascending order, the same for all chunks.
  constexpr int most = moe_most<XT, RT>();
  auto fit = [](int tokens) { return (kMoeLds / (tokens * w4_parts<XT>()) - 16) / (kW4Block * 2); };
  const bool whole = blocks <= fit(min(most, tokens_of_call));
  const Items items(count, groups, 0);
  for (int item = blockIdx.x; item < items.all; item += gridDim.x) {
    const int a = item / items.of_expert, g = (item - a * items.of_expert) * items.rounds, here = min(items.rounds, groups - g);
    const int first = uniform(chosen.first[a]), places = uniform(chosen.first[a + 1]) - first;
    const int expert = uniform(chosen.expert[a]);
    const auto m = matrix((int64_t)expert);
    const W4Rows w[2] = {tile(m, 0), tile(m, 1)};
    for (int p = 0; p < places; p += most) {
      const int tokens = min(most, places - p);
      auto x_of = [&](int t) { return vector(uniform(chosen.place[first + p + t])); };
      // blocks of x at a time: all, or runs that fit
      int chunk = min(blocks, fit(tokens));
      if (chunk < blocks) chunk = chunk / kW4Run * kW4Run;
      const int chunks = (blocks + chunk - 1) / chunk, pitch = chunk * kW4Block * 2 + 16;
      const char* lane_x = lds + w4_row_of_x<w4_parts<XT>()>(w4_thread() % 16, tokens, pitch);
      for (int r = 0; r < here; ++r) {
        const int row = ((g + r) * kMoeWaves + wave) * rows_of_wave;  // (past the end: the last rows again, not stored)
        const int at[2] = {min(first_row(row, 0), w[0].n - 1), min(first_row(row, 1), w[1].n - 1)};
        two.init(w, at, scale_type);
        float sum[2][RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) sum[0][i] = sum[1][i] = 0.f;
        for (int j = 0; j < chunks; ++j) {
          const int start = j * chunk, end = min(start + chunk, full);
          const bool ragged = j == chunks - 1 && full * kW4Block < k;
          typename W4Two<XT, SPB, RT, WIDE, ZEROS>::Ahead ahead;
          // (begins where expert and rows say: which workgroup has them depends on what others have chosen as well)
          const typename W4Two<XT, SPB, RT, WIDE, ZEROS>::Walk walk(start / kW4Run, 1, (end - start + kW4Run - 1) / kW4Run, end,
                                                                    whole ? (unsigned)((expert * groups + g + r) * kMoeWaves + wave) : 0u);
          if (full) two.begin(w[0], walk, ahead);
          if (chunks > 1 || r == 0) {
            __syncthreads();
            w4_stage<XT>(x_of, tokens, k, start, end - start + ragged, lds, pitch, 64 * kMoeWaves);
            __syncthreads();
          }
          two.multiply(w[0], walk, start, ahead, lane_x, pitch, sum);
          if (ragged) two.multiply_tail(w, at, lane_x + (full - start) * kW4Block * 2, pitch, sum);
        }
        const int lane = w4_thread() % 64;
        bool again = false;
#pragma unroll
        for (int i = 0; i < RT; ++i) again |= !(fabsf(sum[0][i]) < INFINITY && fabsf(sum[1][i]) < INFINITY) && lane / 16 + 4 * i < tokens;
        if (__ballot(again)) {
          float plain[2][RT];
#pragma unroll
          for (int i = 0; i < RT; ++i) plain[0][i] = plain[1][i] = 0.f;
#pragma unroll 1
          for (int b = 0; b < blocks; ++b)
            two.block_plain(w, at, b, [&](int i, int l) {
              const int token = min(lane / 16 + 4 * i, tokens - 1);
              return w4_load(XT, vector(chosen.place[first + p + token]), l);
            }, plain);
#pragma unroll
          for (int i = 0; i < 2 * RT; ++i)
            if (!(fabsf(sum[i / RT][i % RT]) < INFINITY)) sum[i / RT][i % RT] = plain[i / RT][i % RT];
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          const int token = lane / 16 + 4 * i;
          if (token < tokens) out(chosen.place[first + p + token], row + lane % 16, sum[0][i], sum[1][i]);
        }
      }
    }
  }
}

// Whether loads of two rows can be made: their second row lies 32 bits from the first.
inline bool moe_fold(const W4Rows& w) {
  constexpr int64_t far = (int64_t)1 << 28;
  return w.k <= kW4Short && w.ld_codes < far && w.ld_scales < far && w.ld_zeros < far;
}
inline int moe_split(int k) {  // waves that share a row, for k up to kMoeLongest
  int log = 0;
  while ((kW4Span << log) < k) ++log;
  return log;
}

}  // namespace
#endif
#endif
