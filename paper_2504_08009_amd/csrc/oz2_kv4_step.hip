// Attention of a few new tokens over a cache held in 4 bits (oz2_kv4_attention): how the work is cut, and how its parts come together.
#include "oz2_kv4_step.h"

extern template hipError_t oz2_kv4_step_of<OZ2_F32>(const Kv4Step&, dim3, hipStream_t);
extern template hipError_t oz2_kv4_step_of<OZ2_BF16>(const Kv4Step&, dim3, hipStream_t);
extern template hipError_t oz2_kv4_step_of<OZ2_F16>(const Kv4Step&, dim3, hipStream_t);

namespace {

// Rows joined: the parts of a row's chunks, each with a maximum of its own, come together: a thread has four dims of every `parts`-th chunk of a row, with a maximum and sums that
// follow as it goes, so that no load waits for another; then the row's `parts` threads of a dim do.  Bound by its waits: the begin, the sequence, the chunks.
// us with all of 256 threads on one row, their maximum looked for first, and so: 4096 rows of up to 8 chunks 12.2 and 6.4, 512 of 8 5.4 and 4.8, 32 of 32 4.6 and 3.9.
struct Finish {
  Kv4Step a;
  FastDiv per_heads, per_pair;
  int shift;              // of the threads that share a row's chunks
  unsigned joins, turns;  // workgroups that join rows; of the others, those of a (sequence, kv head)
};
struct Joining { float sums[256][4], tops[256], totals[256]; };
__device__ __forceinline__ void join(const Finish& f, Joining& sh) {
  const Kv4Step& a = f.a;
  const int parts = 1 << f.shift;
  const int fours = a.dim / 4, thread = threadIdx.x, of = thread / fours, d = (thread - of * fours) * 4, slots = 256 / fours >> f.shift;
  const int slot = of >> f.shift, part = of & (parts - 1);
  const int64_t first = (int64_t)blockIdx.x * slots, row = min(first + slot, a.rows - 1);
  const int begin = (int)first / f.per_heads, at = (int)row / f.per_heads, query = (int)row - at * a.heads;
  const int64_t s = kv_behind(a.on, kv_sequence(a.on.sequences, [&](int64_t i) { return a.on.cu[i] <= begin; }), at);
  const KvRange r = kv_range(a.on.cu, s, a.on.tokens);
  const int held = kv_held(a.on.lengths, s, a.capacity);
  const bool mine = slot < slots && first + slot < a.rows && at >= r.begin && at < r.end && held > a.chunk;
  const int chunks = mine ? (held + a.chunk - 1) / a.chunk : 0;
  const float2* stats = reinterpret_cast<const float2*>(a.stats) + row;
  float high = kNoScore, total = 0.f, v[4] = {};
#pragma unroll 4
  for (int i = part; i < chunks; i += parts) {
    const float2 own = stats[i * a.rows];
    const float4 x = *reinterpret_cast<const float4*>(a.part + (i * a.rows + row) * a.dim + d);
    const float raised = fmaxf(high, own.x), before = __builtin_amdgcn_exp2f(high - raised), now = __builtin_amdgcn_exp2f(own.x - raised);
    total = fmaf(now, own.y, total * before);
    v[0] = fmaf(now, x.x, v[0] * before), v[1] = fmaf(now, x.y, v[1] * before), v[2] = fmaf(now, x.z, v[2] * before), v[3] = fmaf(now, x.w, v[3] * before);
    high = raised;
  }
  if (parts > 1) {
    sh.tops[thread] = high, sh.totals[thread] = total;
    for (int j = 0; j < 4; ++j) sh.sums[thread][j] = v[j];
    __syncthreads();
    if (!mine || part) return;
    float most = high;
    for (int p = 1; p < parts; ++p) most = fmaxf(most, sh.tops[thread + p * fours]);
    float factor = __builtin_amdgcn_exp2f(high - most);
    total *= factor;
    for (int j = 0; j < 4; ++j) v[j] *= factor;
    for (int p = 1; p < parts; ++p) {
      const int from = thread + p * fours;
      factor = __builtin_amdgcn_exp2f(sh.tops[from] - most);
      total = fmaf(factor, sh.totals[from], total);
      for (int j = 0; j < 4; ++j) v[j] = fmaf(factor, sh.sums[from][j], v[j]);
    }
  }
  if (!mine) return;
  for (int j = 0; j < 4; ++j) w4_store(a.out.type, a.out.data, at * a.out.ld_token + query * a.out.ld_head + d + j, total == 0.f ? 0.f : v[j] / total);
}

// What each place received, from the scores and the maxima and sums of its rows, 64 rows at a time and four threads to the chunks of one.  Places that a row does not
// see are passed over, and those on pages that are none altogether: a weight of 0 would be a NaN of a row that is one.
struct Receiving {
  struct alignas(16) Row { float top, scale2, inverse; int sees; const float* scores; } rows[64];
};
__device__ __forceinline__ void receive(const Finish& f, Receiving& sh) {
  const Kv4Step& a = f.a;
  const unsigned i = blockIdx.x - f.joins, pairs = (unsigned)(a.on.sequences * a.c.heads), turn = i / f.per_pair, pair = i - turn * pairs;
  const int s = (int)(pair / (unsigned)a.c.heads), head = (int)(pair - s * (unsigned)a.c.heads), thread = threadIdx.x;
  const int held = kv_held(a.on.lengths, s, a.capacity), chunks = (held + a.chunk - 1) / a.chunk;
  if ((int64_t)turn * 256 >= held) return;
  const KvRange r = kv_range(a.on.cu, s, a.on.tokens);
  const int news = (int)(r.end - r.begin), rows = news * a.group;
  if (!rows) return;
  const int32_t* table = a.on.table + s * a.on.ld_table;
  float* to = a.on.weights + s * a.on.weights_sequence + head * a.on.weights_head;
  for (int64_t first = (int64_t)turn * 256; first < held; first += (int64_t)f.turns * 256) {
    const int place = (int)first + thread, page = place < held ? table[place / a.per_page] : -1;
    const float had = place < held ? to[place] : 0.f;
    float sum = 0.f;
    for (int r0 = 0; r0 < rows; r0 += 64) {
      const int n = min(64, rows - r0), own = r0 + min(thread / 4, n - 1), fresh = own / a.per_group;
      const int64_t row = (r.begin + fresh) * a.heads + head * a.group + (own - fresh * a.group);
      const float2* stats = reinterpret_cast<const float2*>(a.stats) + row;
      float high = kNoScore, total = 0.f;
      auto with = [&](float top, float part) {
        const float raised = fmaxf(high, top);
        total = fmaf(total, __builtin_amdgcn_exp2f(high - raised), part * __builtin_amdgcn_exp2f(top - raised));
        high = raised;
      };
#pragma unroll 4
      for (int c = thread % 4; c < chunks; c += 4) {
        const float2 x = stats[c * a.rows];
        with(x.x, x.y);
      }
      for (int d = 1; d < 4; d *= 2) {
        const float top = __shfl_xor(high, d), part = __shfl_xor(total, d);
        with(top, part);
      }
      __syncthreads();
      if (thread % 4 == 0 && thread / 4 < n) {
        sh.rows[thread / 4] = {high, fabsf(high) > kLarge ? kv_power_above(a.scale2) : a.scale2, total == 0.f ? 0.f : 1.f / total, held - news + fresh + 1, a.scores + row * a.capacity};
      }
      __syncthreads();
      if (place < held) {  // (without a look at the page, so that scores do not wait for it)
#pragma unroll 4
        for (int j = 0; j < n; ++j) {
          const Receiving::Row& x = sh.rows[j];
          const float more = fmaf(__builtin_amdgcn_exp2f(fmaf(x.scores[place], x.scale2, -x.top)), x.inverse, sum);
          sum = place < x.sees ? more : sum;
        }
      }
    }
    if (page >= 0 && page < a.c.pages) to[place] = had + sum;
  }
}

// Both in one launch, side by side: 16 sequences of 2000 to 8192 places and 4 rows, 10.7 us one after the other, 8.3 so.
__global__ void __launch_bounds__(256) kv4_finish_kernel(Finish f) {
  __shared__ union { Joining join; Receiving receive; } sh;
  if (blockIdx.x < f.joins) join(f, sh.join);
  else receive(f, sh.receive);
}

// About a thousand workgroups where there are places enough for them, two rounds of the card; up to 4096 places each, since the begin of a workgroup (some 4 us until
// its first tile is there) is to be spread over enough of them, and no more, since lengths differ.
// us a call with 256 / 1024 / 4096 places (BF16, 8 kv heads of 128): 64 sequences of 2048 to 32768 283 / 188 / 174, 16 of 2000 to 8192 40 / 27 / 40, one of 4096
// 12.3 / 16.7 / 35.7.  What counts is the table's width, which the host knows, not what is held: on one of 131072 places the last two take 39 and 16.9 us instead of 27 and 11.9.
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
  // eighth, which few have (64 sequences of 2048 to 32768 places, 8 kv heads: 292 us a call so, 174 with chunks last, 6 of either to join the parts).
  const dim3 grid((unsigned)cache.heads, (unsigned)on.sequences, (unsigned)chunks);
  hipError_t rc = q.type == OZ2_F32    ? oz2_kv4_step_of<OZ2_F32>(a, grid, st)
                  : q.type == OZ2_BF16 ? oz2_kv4_step_of<OZ2_BF16>(a, grid, st)
                                       : oz2_kv4_step_of<OZ2_F16>(a, grid, st);
  Finish f = {a, fast_div((unsigned)heads), fast_div((unsigned)(on.sequences * cache.heads)), 0, 0, 1};
  if (chunks > 1) {
    // (of rows with few chunks several in a workgroup: about eight chunks for a thread)
    const int64_t most = 256 / (cache.dim / 4);
    while ((2 << f.shift) <= most && chunks > 8 << f.shift) ++f.shift;
    const int64_t slots = most >> f.shift;
    f.joins = (unsigned)((rows + slots - 1) / slots);
  }
  int64_t blocks = f.joins;
  if (on.weights && capacity) {
    const int64_t pairs = on.sequences * cache.heads, turns = (capacity + 255) / 256, most = ((int64_t)1 << 22) / pairs;  // (a grid has fewer than 2^32 threads)
    f.turns = (unsigned)(turns < most ? turns : most);
    blocks += pairs * f.turns;
  }
  if (rc == hipSuccess && blocks) {
    hipLaunchKernelGGL(kv4_finish_kernel, dim3((unsigned)blocks), dim3(256), 0, st, f);
    rc = hipGetLastError();
  }
  return rc;
}
