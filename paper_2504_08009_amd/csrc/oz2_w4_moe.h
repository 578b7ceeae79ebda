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
  hipStream_t st;
};

W4Rows oz2_w4_rows(const oz2_w4_matrix& m);
template <int XT>
hipError_t oz2_moe_gate_up(const MoeCall& c, int scale_type);
hipError_t oz2_moe_down(const MoeCall& c, int scale_type);
int oz2_w4_compute_units();

#ifdef __HIPCC__
namespace {

constexpr int kMoeWaves = 8, kMoeRounds = 8;

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

// Rows of experts times the places that chose them.  A workgroup takes an item (an expert and `rounds` batches of its rows) after the other; a batch
// is four rows of codes for each `1 << split_log` waves.  row(expert's matrices, i): the i-th row of the batch at that row; x(place): vector.
// out(place, batch's row, sums of the four rows): called by one thread.
template <int XT, int T, int ST, bool ZEROS, class Matrix, class Row, class X, class Out>
__device__ __forceinline__ void moe_products(const Chosen& chosen, int k, int rows, int rows_of_batch, int split_log, const W4Rows& shape, float (*part)[kMoeRounds][kMoeWaves][4][T],
                                             Matrix matrix, Row row_of, X vector, Out out) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int split = 1 << split_log, s = wave & (split - 1), group = wave >> split_log, per = kMoeWaves >> split_log;
  const int unit = s * 64 + lane;
  const W4Place at = w4_place(shape, unit);
  const bool ragged = __ballot(at.cut != 0) != 0;
  // as many rounds as leave every workgroup two items or more
  const int batches = (rows + rows_of_batch * per - 1) / (rows_of_batch * per);
  auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int count = uniform(chosen.count);
  int rounds = min(kMoeRounds, max(1, (int)((int64_t)batches * count / (2 * gridDim.x))));
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
      W4Rows4<XT, T, ST, ZEROS> r;
      r.fetch(rows_at(0), at);
      W4X<XT> kept[T];
      const unsigned plain = w4_take_x<XT, T>(k, unit, x_at, kept);
      for (int i = 0; i < turns; ++i) {
        float sum[4][T];
        r.multiply(at, kept, ragged, sum);
        if (plain) r.multiply_plain(plain, k, shape.group, rows_at(i), x_at, unit, sum);
        if (i + 1 < turns) r.fetch(rows_at(i + 1), at);
        float v[T];
#pragma unroll
        for (int t = 0; t < T; ++t) v[t] = w4_sum4(sum[0][t], sum[1][t], sum[2][t], sum[3][t]);
        const int t = lane % 16;
        if (t < T) part[flip][i][wave][lane / 16][t] = T == 2 && t ? v[T - 1] : v[0];
      }
      __syncthreads();
      for (int j = threadIdx.x; j < turns * per * T; j += 64 * kMoeWaves) {
        const int t = j % T, g = j / T % per, i = j / T / per;
        if (p + t >= places) continue;
        float u[4] = {0.f, 0.f, 0.f, 0.f};
        for (int q = 0; q < split; ++q)
#pragma unroll
          for (int n = 0; n < 4; ++n) u[n] += part[flip][i][g * split + q][n][t];
        out(chosen.place[first + p + t], (start + i * per + g) * rows_of_batch, u);
      }
      flip ^= 1;
    }
  }
}

inline int moe_split(int k) {
  int log = 0;
  while ((kW4Span << log) < k) ++log;
  return log;
}

}  // namespace
#endif
#endif
