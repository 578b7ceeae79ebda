// Eviction from a cache held in 4 bits (oz2_kv4_evict), in two launches: a workgroup chooses for each sequence and kv head, then many move tokens.
//
// The choice: an unsigned key that orders weights as oz2.h says; the keep-th largest key by four passes over eight bits each, from the top, with a histogram in
// LDS (sixteen copies, since most weights share a few exponents and additions to one word wait for each other); places with that key itself are taken from the lowest on.  Places
// below `keep` that were given up and places from `keep` on that stay are then listed in order by prefix sums over the threads, each of which has a run of
// places.
#include "oz2_kv4.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kCopies = 16;
constexpr unsigned kStays = ~0u, kNan = ~0u - 1;

struct Evict {
  oz2_kv4_cache c;
  oz2_kv4_sequences on;
  oz2_kv4_kept to;
  int capacity, keep, recent, most;  // most: moves that a head can have
  int32_t *count, *from, *into;      // of (sequence, head); most of each
};

struct Shared {
  unsigned bins[256 * kCopies];
  unsigned wave[kWaves], wave2[kWaves];
  int newest[kWaves];
  unsigned prefix, left;
};

__device__ __forceinline__ unsigned key_of(float w, int position, int64_t newest, int recent) {
  if ((int64_t)position > newest - recent) return kStays;
  if (w != w) return kNan;
  const unsigned b = __float_as_uint(w + 0.f);  // (-0 is 0)
  return b ^ (b >> 31 ? ~0u : 0x80000000u);
}

// Sum of v over the threads before this one, of two numbers at once; every thread calls it.
__device__ __forceinline__ uint2 before(uint2 v, Shared& sh) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  uint2 sum = v;
  for (int d = 1; d < 64; d *= 2) {
    const unsigned x = __shfl_up(sum.x, d), y = __shfl_up(sum.y, d);
    if (lane >= d) sum.x += x, sum.y += y;
  }
  __syncthreads();
  if (lane == 63) sh.wave[wave] = sum.x, sh.wave2[wave] = sum.y;
  __syncthreads();
  uint2 base = {0, 0};
  for (int i = 0; i < wave; ++i) base.x += sh.wave[i], base.y += sh.wave2[i];
  return {base.x + sum.x - v.x, base.y + sum.y - v.y};
}

__global__ void __launch_bounds__(kThreads) kv4_choose_kernel(Evict a) {
  __shared__ Shared sh;
  const int heads = (int)a.c.heads, s = blockIdx.x / heads, head = blockIdx.x % heads;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int held = kv_held(a.on.lengths, s, a.capacity);
  const int32_t* positions = a.on.positions + s * a.on.positions_sequence + head * a.on.positions_head;
  const float* weights = a.on.weights + s * a.on.weights_sequence + head * a.on.weights_head;
  int32_t* to_positions = a.to.positions + s * a.to.positions_sequence + head * a.to.positions_head;
  float* to_weights = a.to.weights + s * a.to.weights_sequence + head * a.to.weights_head;
  if (held <= a.keep || a.keep == 0) {
    if (threadIdx.x == 0) a.count[blockIdx.x] = 0;
    for (int t = threadIdx.x; t < held && t < a.keep; t += kThreads) {
      if (to_positions != positions) to_positions[t] = positions[t];
      if (to_weights != weights) to_weights[t] = weights[t];
    }
    return;
  }

  int newest = INT32_MIN;
  for (int t = threadIdx.x; t < held; t += kThreads) newest = max(newest, positions[t]);
  for (int d = 32; d; d /= 2) newest = max(newest, __shfl_xor(newest, d));
  if (lane == 0) sh.newest[wave] = newest;
  __syncthreads();
  for (int i = 0; i < kWaves; ++i) newest = max(newest, sh.newest[i]);

  // the keep-th largest key, and how many of those that equal it stay
  unsigned prefix = 0, left = a.keep;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256 * kCopies; i += kThreads) sh.bins[i] = 0;
    __syncthreads();
    for (int t = threadIdx.x; t < held; t += kThreads) {
      const unsigned k = key_of(weights[t], positions[t], newest, a.recent);
      if (shift == 24 || k >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&sh.bins[(k >> shift & 255) * kCopies + lane % kCopies], 1u);
    }
    __syncthreads();
    if (wave == 0) {  // bins from the top: lane l has 255 - 4 l and the three below
      unsigned n[4], sum = 0;
      for (int j = 0; j < 4; ++j) {
        n[j] = 0;
        for (int i = 0; i < kCopies; ++i) n[j] += sh.bins[(255 - 4 * lane - j) * kCopies + (i + lane) % kCopies];
        sum += n[j];
      }
      unsigned upto = sum;
      for (int d = 1; d < 64; d *= 2) {
        const unsigned x = __shfl_up(upto, d);
        if (lane >= d) upto += x;
      }
      unsigned above = upto - sum;
      if (above < left && upto >= left) {  // one lane
        for (int j = 0; j < 4; ++j) {
          if (above < left && above + n[j] >= left) {
            sh.prefix = prefix | (unsigned)(255 - 4 * lane - j) << shift;
            sh.left = left - above;
            break;
          }
          above += n[j];
        }
      }
    }
    __syncthreads();
    prefix = sh.prefix, left = sh.left;
  }

  const int run = (held + kThreads - 1) / kThreads, first = min((int)threadIdx.x * run, held), last = min(first + run, held);
  unsigned ties = 0;
  for (int t = first; t < last; ++t) ties += key_of(weights[t], positions[t], newest, a.recent) == prefix;
  const unsigned ties_before = before({ties, 0}, sh).x;
  int32_t* from = a.from + (int64_t)blockIdx.x * a.most;
  int32_t* into = a.into + (int64_t)blockIdx.x * a.most;
  uint2 n = {0, 0}, at = {0, 0};
  for (int pass = 0; pass < 2; ++pass) {
    unsigned tie = ties_before;
    uint2 i = at;
    for (int t = first; t < last; ++t) {
      const unsigned k = key_of(weights[t], positions[t], newest, a.recent);
      const bool stays = k > prefix || (k == prefix && tie < left);
      tie += k == prefix;
      if (t < a.keep) {
        if (!stays) {
          if (pass) into[i.x] = t;
          ++i.x;
        }
      } else if (stays) {
        if (pass) from[i.y] = t;
        ++i.y;
      }
    }
    if (!pass) {
      n = i;
      at = before(n, sh);
    }
  }
  if (threadIdx.x == kThreads - 1) sh.prefix = at.x + n.x;
  __syncthreads();
  const int count = (int)sh.prefix;
  if (threadIdx.x == 0) a.count[blockIdx.x] = count;
  // (no place is both read and written: what moves comes from `keep` on)
  if (to_positions != positions)
    for (int t = threadIdx.x; t < a.keep; t += kThreads) to_positions[t] = positions[t];
  if (to_weights != weights)
    for (int t = threadIdx.x; t < a.keep; t += kThreads) to_weights[t] = weights[t];
  __syncthreads();
  for (int i = threadIdx.x; i < count; i += kThreads) {
    const int f = from[i], t = into[i];
    to_positions[t] = positions[f];
    to_weights[t] = weights[f];
  }
}

__global__ void __launch_bounds__(256) kv4_move_kernel(Evict a, int lanes) {
  const int heads = (int)a.c.heads, s = blockIdx.x / heads, head = blockIdx.x % heads;
  if (blockIdx.y == 0 && head == 0 && threadIdx.x == 0) a.to.lengths[s] = min(kv_held(a.on.lengths, s, a.capacity), a.keep);
  const int count = a.count[blockIdx.x], lane = threadIdx.x % lanes, per = 256 / lanes;
  const int32_t* from = a.from + (int64_t)blockIdx.x * a.most;
  const int32_t* into = a.into + (int64_t)blockIdx.x * a.most;
  const int page_size = (int)a.c.page_size, row = (int)a.c.dim / 2;
  for (int i = blockIdx.y * per + threadIdx.x / lanes; i < count; i += gridDim.y * per) {
    const int f = from[i], t = into[i];
    const int64_t fp = a.on.table[s * a.on.ld_table + f / page_size], tp = a.on.table[s * a.on.ld_table + t / page_size];
    if (fp < 0 || fp >= a.c.pages || tp < 0 || tp >= a.c.pages) continue;
    const int64_t fc = fp * a.c.codes_page + head * a.c.codes_head + (int64_t)(f % page_size) * row, tc = tp * a.c.codes_page + head * a.c.codes_head + (int64_t)(t % page_size) * row;
    if (lane * 4 < row) {
      *reinterpret_cast<unsigned*>(a.c.k_codes + tc + lane * 4) = *reinterpret_cast<const unsigned*>(a.c.k_codes + fc + lane * 4);
      *reinterpret_cast<unsigned*>(a.c.v_codes + tc + lane * 4) = *reinterpret_cast<const unsigned*>(a.c.v_codes + fc + lane * 4);
    }
    if (lane == 0) {
      const int64_t fs = fp * a.c.scales_page + head * a.c.scales_head + f % page_size, ts = tp * a.c.scales_page + head * a.c.scales_head + t % page_size;
      static_cast<unsigned*>(a.c.k_scales)[ts] = static_cast<const unsigned*>(a.c.k_scales)[fs];
      static_cast<unsigned*>(a.c.v_scales)[ts] = static_cast<const unsigned*>(a.c.v_scales)[fs];
    }
  }
}

int64_t moves(const oz2_kv4_cache& cache, int64_t max_pages, int64_t keep) {
  const int64_t capacity = max_pages * cache.page_size;
  return capacity <= keep ? 0 : keep < capacity - keep ? keep : capacity - keep;
}
int64_t counts(const oz2_kv4_cache& cache, int64_t sequences) { return (sequences * cache.heads + 63) / 64 * 64; }

}  // namespace

size_t oz2_kv4_evict_space(const oz2_kv4_cache& cache, int64_t sequences, int64_t max_pages, int64_t keep) {
  return (size_t)(counts(cache, sequences) + 2 * sequences * cache.heads * moves(cache, max_pages, keep)) * 4;
}

hipError_t oz2_launch_kv4_evict(const oz2_kv4_cache& cache, const oz2_kv4_sequences& on, int64_t keep, int64_t recent, const oz2_kv4_kept& to, char* ws,
                                hipStream_t st) {
  const int64_t capacity = on.max_pages * cache.page_size, all = on.sequences * cache.heads, most = moves(cache, on.max_pages, keep);
  int32_t* count = reinterpret_cast<int32_t*>(ws);
  int32_t* from = count + counts(cache, on.sequences);
  const Evict a = {cache, on, to, (int)capacity, (int)(keep < capacity ? keep : capacity), (int)(recent < capacity ? recent : capacity), (int)most, count, from,
                   from + all * most};
  hipLaunchKernelGGL(kv4_choose_kernel, dim3((unsigned)all), dim3(kThreads), 0, st, a);
  const hipError_t rc = hipGetLastError();
  if (rc != hipSuccess) return rc;
  int lanes = 1;
  while (lanes * 8 < cache.dim) lanes *= 2;
  const int64_t blocks = (most * lanes + 255) / 256;
  hipLaunchKernelGGL(kv4_move_kernel, dim3((unsigned)all, (unsigned)(blocks < 1 ? 1 : blocks < 256 ? blocks : 256)), dim3(256), 0, st, a, lanes);
  return hipGetLastError();
}
