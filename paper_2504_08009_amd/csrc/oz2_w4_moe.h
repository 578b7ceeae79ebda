// A layer of gated experts held in 4 bits (oz2_w4_moe): what its kernels share.  Dispatch in oz2_w4_moe.hip, the products with the
// experts by type of the tokens in oz2_w4_moe_f32.hip, oz2_w4_moe_bf16.hip, oz2_w4_moe_f16.hip, the second ones in oz2_w4_moe_down.hip.
#ifndef OZ2_W4_MOE_H
#define OZ2_W4_MOE_H

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
  int pairs;        // 1: two tokens of an expert at a time, 0: one
  hipStream_t st;
};

W4Rows oz2_w4_rows(const oz2_w4_matrix& m);
template <int XT>
hipError_t oz2_moe_gate_up(const MoeCall& c, int scale_type);
hipError_t oz2_moe_down(const MoeCall& c, int scale_type);
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

struct MoeItem {
  int expert, first, places, row;
};

__device__ __forceinline__ W4Rows w4_of_stack(W4Rows w, int64_t e, int64_t codes, int64_t scales, int64_t zeros) {
  w.codes += e * codes, w.scales += e * scales, w.zeros += e * zeros;
  return w;
}

// Rows of experts times the places that chose them.  A workgroup takes an item (an expert and up to kMoeRounds batches of its rows) after the other;
// a batch is four loads of rows for each `1 << split_log` waves, `loads` of which (4, or 2 beside 2 of a second matrix) are of one matrix.
// row(expert's matrices, row, i): the i-th load of the batch from that row; x(place): vector; out(place, row, sums): called by one
// thread with the sums of the batch's 4 FOLD rows.
template <int XT, int T, int ST, bool ZEROS, int FOLD, class Matrix, class Row, class X, class Out>
__device__ __forceinline__ void moe_products(const Chosen& chosen, int k, int rows, int loads, int split_log, const W4Rows& shape,
                                             float (*part)[kMoeRounds][kMoeWaves][4 * FOLD][T], Matrix matrix, Row row_of, X vector, Out out) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int split = 1 << split_log, s = wave & (split - 1), group = wave >> split_log, per = kMoeWaves >> split_log;
  const int unit = FOLD == 2 ? lane % 32 : s * 64 + lane, rows_of_batch = loads * FOLD;
  const W4Place at = w4_place(shape, unit);
  const bool ragged = __ballot(at.cut != 0) != 0;
  auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int count = uniform(chosen.count);
  // as many rounds as leave every workgroup one item, if that can be
  const int batches = (rows + rows_of_batch * per - 1) / (rows_of_batch * per);
  const int rounds = max(1, min(kMoeRounds, (batches * count + (int)gridDim.x - 1) / (int)gridDim.x));
  const int chunks = (batches + rounds - 1) / rounds;
  int flip = 0;
  for (int item = blockIdx.x; item < count * chunks; item += gridDim.x) {
    const int a = item / chunks, chunk = item - a * chunks;
    const int first = uniform(chosen.first[a]), places = uniform(chosen.first[a + 1]) - first;
    const auto m = matrix((int64_t)uniform(chosen.expert[a]));
    const int start = chunk * rounds * per, turns = min(rounds, batches - chunk * rounds);
    auto rows_at = [&](int i) {
      const int row = (start + i * per + group) * rows_of_batch;
      return [&, row](int j) { return row_of(m, row, j); };
    };
    for (int p = 0; p < places; p += T) {
      auto x_at = [&](int t) { return vector(uniform(chosen.place[first + min(p + t, places - 1)])); };
      W4Rows4<XT, T, ST, ZEROS, FOLD> r;
      r.fetch(rows_at(0), at);
      W4X<XT> kept[T];
      const unsigned plain = w4_take_x<XT, T>(k, unit, x_at, kept);
      for (int i = 0; i < turns; ++i) {
        float sum[4][T];
        r.multiply(at, kept, ragged, sum);
        if (plain) r.multiply_plain(plain, k, shape.group, rows_at(i), x_at, unit, sum);
        if (i + 1 < turns) r.fetch(rows_at(i + 1), at);
#pragma unroll
        for (int t = 0; t < T; ++t) {
          float v[FOLD];
          w4_sum4<FOLD>(sum[0][t], sum[1][t], sum[2][t], sum[3][t], v);
          if (lane % 16 == 0)
#pragma unroll
            for (int j = 0; j < FOLD; ++j) part[flip][i][wave][w4_row_of_lane<FOLD>(j)][t] = v[j];
        }
      }
      __syncthreads();
      for (int j = threadIdx.x; j < turns * per * T; j += 64 * kMoeWaves) {
        const int t = j % T, g = j / T % per, i = j / T / per;
        if (p + t >= places) continue;
        float u[4 * FOLD];
#pragma unroll
        for (int n = 0; n < 4 * FOLD; ++n) u[n] = part[flip][i][g * split][n][t];
        for (int q = 1; q < split; ++q)
#pragma unroll
          for (int n = 0; n < 4 * FOLD; ++n) u[n] += part[flip][i][g * split + q][n][t];
        out(chosen.place[first + p + t], (start + i * per + g) * rows_of_batch, u);
      }
      flip ^= 1;
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
