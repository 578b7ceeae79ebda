// Attention of a few new tokens over a cache held in 4 bits (oz2_kv4_attention): how the work is cut, and how its parts come together.
#include "oz2_kv4_step.h"

extern template hipError_t oz2_kv4_step_of<OZ2_F32>(const Kv4Step&, dim3, hipStream_t);
extern template hipError_t oz2_kv4_step_of<OZ2_BF16>(const Kv4Step&, dim3, hipStream_t);
extern template hipError_t oz2_kv4_step_of<OZ2_F16>(const Kv4Step&, dim3, hipStream_t);

namespace {

// A workgroup a row: the parts of its chunks, each with a maximum of its own.  A thread has four dims of every 1024 / dim-th chunk.
__global__ void __launch_bounds__(256) kv4_join_kernel(Kv4Step a, FastDiv per_heads) {
  __shared__ float factor[256], sums[256][4], most[4], totals[4];
  const int row = blockIdx.x, at = row / per_heads, query = row - at * a.heads, thread = threadIdx.x, lane = thread % 64, wave = thread / 64;
  const int64_t token = at, s = kv_sequence(a.on.sequences, [&](int64_t i) { return a.on.cu[i] <= token; });
  const KvRange r = kv_range(a.on.cu, s, a.on.tokens);
  if (token < r.begin || token >= r.end) return;
  const int held = kv_held(a.on.lengths, s, a.capacity);
  if (held <= a.chunk) return;
  const int chunks = (held + a.chunk - 1) / a.chunk;
  const float2* stats = reinterpret_cast<const float2*>(a.stats) + row;
  float high = -3e38f;
  for (int i = thread; i < chunks; i += 256) high = fmaxf(high, stats[i * a.rows].x);
  for (int d = 32; d; d /= 2) high = fmaxf(high, __shfl_xor(high, d));
  if (lane == 0) most[wave] = high;
  __syncthreads();
  high = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
  const int fours = a.dim / 4, part = thread / fours, parts = 256 / fours, d = thread % fours * 4;
  float total = 0.f, v[4] = {};
  for (int c0 = 0; c0 < chunks; c0 += 256) {
    const int n = min(256, chunks - c0);
    __syncthreads();
    if (thread < n) {
      const float2 own = stats[(c0 + thread) * a.rows];
      factor[thread] = __builtin_amdgcn_exp2f(own.x - high);
      total = fmaf(factor[thread], own.y, total);
    }
    __syncthreads();
    if (part < parts) {
#pragma unroll 4
      for (int i = part; i < n; i += parts) {
        const float4 x = *reinterpret_cast<const float4*>(a.part + ((c0 + i) * a.rows + row) * a.dim + d);
        v[0] = fmaf(factor[i], x.x, v[0]), v[1] = fmaf(factor[i], x.y, v[1]), v[2] = fmaf(factor[i], x.z, v[2]), v[3] = fmaf(factor[i], x.w, v[3]);
      }
    }
  }
  for (int i = 32; i; i /= 2) total += __shfl_xor(total, i);
  if (lane == 0) totals[wave] = total;
  for (int j = 0; j < 4; ++j) sums[thread][j] = v[j];
  __syncthreads();
  if (part) return;
  total = totals[0] + totals[1] + totals[2] + totals[3];
  if (thread == 0) const_cast<float2*>(stats)[0] = {high, total};  // the whole row's, in the place of its first chunk's: kv4_received_kernel reads them
  for (int p = 1; p < parts; ++p)
    for (int j = 0; j < 4; ++j) v[j] += sums[p * fours + thread][j];
  for (int j = 0; j < 4; ++j) w4_store(a.out.type, a.out.data, token * a.out.ld_token + query * a.out.ld_head + d + j, total == 0.f ? 0.f : v[j] / total);
}

// What each place received, from the scores and the rows' maxima and sums, which are in the places of their first chunks.
__global__ void __launch_bounds__(256) kv4_received_kernel(Kv4Step a) {
  __shared__ float top[64], inverse[64];
  __shared__ const float* scores[64];
  const int head = blockIdx.x, s = blockIdx.y, place = blockIdx.z * 256 + threadIdx.x;
  const int held = kv_held(a.on.lengths, s, a.capacity);
  if ((int)blockIdx.z * 256 >= held) return;
  const KvRange r = kv_range(a.on.cu, s, a.on.tokens);
  const int rows = (int)(r.end - r.begin) * a.group;
  float* to = a.on.weights + s * a.on.weights_sequence + head * a.on.weights_head + place;
  const float had = rows && place < held ? *to : 0.f;
  float sum = 0.f;
  for (int r0 = 0; r0 < rows; r0 += 64) {
    __syncthreads();
    const int n = min(64, rows - r0);
    if ((int)threadIdx.x < n) {
      const int fresh = (int)(r0 + threadIdx.x) / a.per_group;
      const int64_t row = (r.begin + fresh) * a.heads + head * a.group + (r0 + (int)threadIdx.x - fresh * a.group);
      const float total = a.stats[row * 2 + 1];
      top[threadIdx.x] = a.stats[row * 2];
      inverse[threadIdx.x] = total == 0.f ? 0.f : 1.f / total;
      scores[threadIdx.x] = a.scores + row * a.capacity;
    }
    __syncthreads();
    if (place < held) {
#pragma unroll 4
      for (int i = 0; i < n; ++i) sum = fmaf(__builtin_amdgcn_exp2f(fmaf(scores[i][place], a.scale2, -top[i])), inverse[i], sum);
    }
  }
  if (rows && place < held) *to = had + sum;
}

// About a thousand workgroups where there are places enough for them, two rounds of the card; up to 4096 places each, since the begin of a workgroup (some 4 us until
// its first tile is there) is to be spread over enough of them, and no more, since lengths differ.
// us with 256 / 1024 / 4096 places: 64 sequences of 2048 to 32768 360 / 213 / 183, 16 of 2000 to 8192 47 / 36 / 46, one of 4096 (8 kv heads) 8 / 14 / 36.
int64_t chunk_of(int64_t capacity, int64_t pairs) {
  const int64_t each = (capacity * pairs + 1023) / 1024;
  const int64_t chunk = (each + 127) / 128 * 128;
  return chunk < 128 ? 128 : chunk < 4096 ? chunk : 4096;
}
size_t rounded(int64_t n) { return (size_t)((n + 63) / 64 * 64) * 4; }
struct Space { size_t part, stats, scores; };
Space space(int64_t capacity, int64_t chunk, int64_t rows, int64_t dim, bool weights) {
  const int64_t chunks = (capacity + chunk - 1) / chunk;
  return {chunks > 1 ? rounded(chunks * rows * dim) : 0, chunks > 1 || weights ? rounded(chunks * rows * 2) : 0, weights ? rounded(rows * capacity) : 0};
}

}  // namespace

size_t oz2_kv4_attention_space(const oz2_kv4_cache& cache, int64_t sequences, int64_t max_pages, int64_t tokens, int64_t heads, int weights) {
  const int64_t capacity = max_pages * cache.page_size;
  const Space n = space(capacity, chunk_of(capacity, sequences * cache.heads), tokens * heads, cache.dim, weights != 0);
  return n.part + n.stats + n.scores;
}

hipError_t oz2_launch_kv4_attention(const oz2_kv4_cache& cache, const oz2_kv4_sequences& on, int64_t heads, float scale, const oz2_rows& q,
                                    const oz2_rows& out, char* ws, hipStream_t st) {
  const int64_t capacity = on.max_pages * cache.page_size, chunk = chunk_of(capacity, on.sequences * cache.heads), rows = on.tokens * heads;
  const int64_t chunks = capacity ? (capacity + chunk - 1) / chunk : 1;
  const Space n = space(capacity, chunk, rows, cache.dim, on.weights != nullptr);
  Kv4Step a = {};
  a.c = cache, a.on = on, a.q = q, a.out = out;
  a.heads = (int)heads, a.group = (int)(heads / cache.heads), a.dim = (int)cache.dim, a.capacity = (int)capacity;
  a.page_size = (int)cache.page_size, a.chunk = (int)chunk;
  a.per_page = fast_div((unsigned)cache.page_size), a.per_group = fast_div((unsigned)a.group);
  a.scale2 = (float)(scale * 1.4426950408889634074) * (q.type == OZ2_F32 ? step_score<OZ2_F32>() : step_score<OZ2_BF16>());
  a.part = n.part ? reinterpret_cast<float*>(ws) : nullptr;
  a.stats = n.stats ? reinterpret_cast<float*>(ws + n.part) : nullptr;
  a.scores = n.scores ? reinterpret_cast<float*>(ws + n.part + n.stats) : nullptr;
  a.rows = rows;
  // Chunks last: eight dies take workgroups in turn, and with chunks first one of them would get all first chunks, which every sequence has, and another the
  // eighth, which few have (64 sequences of 2048 to 32768 places, 8 kv heads: 355 us so, 150 with chunks last).
  const dim3 grid((unsigned)cache.heads, (unsigned)on.sequences, (unsigned)chunks);
  hipError_t rc = q.type == OZ2_F32    ? oz2_kv4_step_of<OZ2_F32>(a, grid, st)
                  : q.type == OZ2_BF16 ? oz2_kv4_step_of<OZ2_BF16>(a, grid, st)
                                       : oz2_kv4_step_of<OZ2_F16>(a, grid, st);
  if (rc == hipSuccess && chunks > 1) {
    hipLaunchKernelGGL(kv4_join_kernel, dim3((unsigned)rows), dim3(256), 0, st, a, fast_div((unsigned)heads));
    rc = hipGetLastError();
  }
  if (rc == hipSuccess && on.weights && capacity) {
    hipLaunchKernelGGL(kv4_received_kernel, dim3((unsigned)cache.heads, (unsigned)on.sequences, (unsigned)((capacity + 255) / 256)), dim3(256), 0, st, a);
    rc = hipGetLastError();
  }
  return rc;
}
