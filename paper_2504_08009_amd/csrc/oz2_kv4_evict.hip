// Eviction from a cache held in 4 bits (oz2_kv4_evict): a workgroup chooses for each sequence and kv head, then many move tokens, or the same one where they are few.
//
// The choice: an unsigned key that orders weights as oz2.h says; the keep-th largest key by three passes over its bits from the top, with a histogram of 2048
// bins in LDS; places with that key itself are taken from the lowest on.  Places below `keep` that were given up and places from `keep` on that stay are then
// listed in order, by ranks from the lanes' votes.  Bound by the waits between these steps, and by what one compute unit reads, 8 bytes a place: of 64 heads with up to
// 32768 places and 4096 to keep, 8 us until the keys are there, 2 for the recent ones, 8 for the passes, 7 for the ranks; the moves, rows of 64 bytes from anywhere, 20.
#include "oz2_kv4.h"
#include "oz2_fast_div.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kFew = 256, kAtOnce = 4;
constexpr unsigned kStays = ~0u, kNan = ~0u - 1;

struct Evict {
  oz2_kv4_cache c;
  oz2_kv4_sequences on;
  oz2_kv4_kept to;
  int capacity, keep, recent, most;  // most: moves that a head can have
  int page_size, heads_count, lanes; // lanes a token is moved by
  FastDiv per_page, heads;
  int32_t *count, *from, *into;      // of (sequence, head); most of each
};

constexpr int kBins = 2048;
struct Shared {
  unsigned bins[kBins * 2];  // two copies each
  unsigned wave[kWaves], wave2[kWaves];
  int newest;
  unsigned prefix, left, equal, total;
};

__device__ __forceinline__ unsigned key_of(float w) {
  if (w != w) return kNan;
  const unsigned b = __float_as_uint(w + 0.f);  // (-0 is 0)
  return b ^ (b >> 31 ? ~0u : 0x80000000u);
}
__device__ __forceinline__ unsigned key_of(float w, int position, int64_t newest, int recent) {
  return (int64_t)position > newest - recent ? kStays : key_of(w);
}

// Sum of v over the lanes up to this one: shifts within rows of sixteen lanes, then the rows' last lanes to the rows behind.
__device__ __forceinline__ unsigned upto_lane(unsigned v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}
// Sum of the waves' numbers before wave `wave`, from sixteen of them in LDS.
__device__ __forceinline__ unsigned before_wave(const unsigned* of_wave, int wave) {
  const int lane = threadIdx.x % 64;
  return wave ? (unsigned)__builtin_amdgcn_readlane((int)upto_lane(lane < kWaves ? of_wave[lane] : 0), wave - 1) : 0u;
}

struct Choice { unsigned prefix, left, equal; };  // a key, how many that equal it stay, and how many there are

// The keep-th largest of the keys (0: none) that each(f) shows to f, thread by thread the same ones at every call: eleven, eleven and ten bits, from the top.
template <class Each>
__device__ __forceinline__ Choice choice(int keep, Shared& sh, Each each) {
  const int thread = threadIdx.x, lane = thread % 64, wave = __builtin_amdgcn_readfirstlane(thread / 64);
  Choice c = {0, (unsigned)keep, 0};
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, upper = pass == 0 ? 32 : pass == 1 ? 21 : 10;
    const unsigned digit = (1u << (upper - shift)) - 1;
    reinterpret_cast<uint4*>(sh.bins)[thread] = uint4{0, 0, 0, 0};
    __syncthreads();
    each([&](unsigned k) {
      if (k && (pass == 0 || (k ^ c.prefix) >> (upper % 32) == 0)) atomicAdd(&sh.bins[(k >> shift & digit) * 2 + lane % 2], 1u);
    });
    __syncthreads();
    // bins from the top: a thread has 2047 - 2 thread and the one below
    const uint4 n4 = reinterpret_cast<const uint4*>(sh.bins)[kThreads - 1 - thread];
    const unsigned n[2] = {n4.z + n4.w, n4.x + n4.y};
    const unsigned upto = upto_lane(n[0] + n[1]);
    if (lane == 63) sh.wave[wave] = upto;
    __syncthreads();
    unsigned above = upto - n[0] - n[1] + before_wave(sh.wave, wave);
    for (int j = 0; j < 2; ++j) {
      if (above < c.left && above + n[j] >= c.left) {  // one thread
        sh.prefix = c.prefix | (unsigned)(kBins - 1 - 2 * thread - j) << shift;
        sh.left = c.left - above;
        sh.equal = n[j];
        break;
      }
      above += n[j];
    }
    __syncthreads();
    c = {sh.prefix, sh.left, sh.equal};
  }
  return c;
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

// Copies tokens f[i] of a sequence and head to places t[i] (where f[i] is not negative): `lane` has eight codes of the keys and of the values, lane 0 the scales too.
// N tokens at once: each takes three trips to memory, one behind the other.
template <int N>
__device__ __forceinline__ void move(const Evict& a, int s, int head, const int (&f)[N], const int (&t)[N], int lane) {
  const int row = (int)a.c.dim / 2;
  int64_t fp[N], tp[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    fp[i] = f[i] < 0 ? -1 : a.on.table[s * a.on.ld_table + f[i] / a.per_page];
    tp[i] = f[i] < 0 ? -1 : a.on.table[s * a.on.ld_table + t[i] / a.per_page];
  }
  unsigned k[N], v[N], ks[N], vs[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (fp[i] < 0 || fp[i] >= a.c.pages || tp[i] < 0 || tp[i] >= a.c.pages) {
      tp[i] = -1;
      continue;
    }
    const int in = f[i] - f[i] / a.per_page * a.page_size;
    if (lane * 4 < row) {
      const int64_t at = fp[i] * a.c.codes_page + head * a.c.codes_head + (int64_t)in * row + lane * 4;
      k[i] = *reinterpret_cast<const unsigned*>(a.c.k_codes + at);
      v[i] = *reinterpret_cast<const unsigned*>(a.c.v_codes + at);
    }
    if (lane == 0) {
      const int64_t at = fp[i] * a.c.scales_page + head * a.c.scales_head + in;
      ks[i] = static_cast<const unsigned*>(a.c.k_scales)[at];
      vs[i] = static_cast<const unsigned*>(a.c.v_scales)[at];
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (tp[i] < 0) continue;
    const int in = t[i] - t[i] / a.per_page * a.page_size;
    if (lane * 4 < row) {
      const int64_t at = tp[i] * a.c.codes_page + head * a.c.codes_head + (int64_t)in * row + lane * 4;
      *reinterpret_cast<unsigned*>(a.c.k_codes + at) = k[i];
      *reinterpret_cast<unsigned*>(a.c.v_codes + at) = v[i];
    }
    if (lane == 0) {
      const int64_t at = tp[i] * a.c.scales_page + head * a.c.scales_head + in;
      static_cast<unsigned*>(a.c.k_scales)[at] = ks[i];
      static_cast<unsigned*>(a.c.v_scales)[at] = vs[i];
    }
  }
}

// Four values beside each other.
template <class T>
__device__ __forceinline__ void four(const T* p, T (&x)[4]) {
  struct __attribute__((packed, aligned(4))) Four { T v[4]; };
  const Four f = *reinterpret_cast<const Four*>(p);
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = f.v[j];
}

// PLACES: most that a sequence holds, whose keys lie in LDS (0: no place, which no key is).  MOVES: the tokens are moved here too.
template <int PLACES, bool MOVES>
__global__ void __launch_bounds__(kThreads) kv4_choose_kernel(Evict a) {
  __shared__ Shared sh;
  __shared__ uint4 keys[PLACES / 4];
  __shared__ unsigned counts[PLACES / 256];  // of 256 places each, which a wave looks at at a time
  const int s = blockIdx.x / a.heads, head = blockIdx.x - s * a.heads_count;
  const int thread = threadIdx.x, lane = thread % 64, wave = __builtin_amdgcn_readfirstlane(thread / 64);
  const int held = kv_held(a.on.lengths, s, a.capacity);
  const int32_t* positions = a.on.positions + s * a.on.positions_sequence + head * a.on.positions_head;
  const float* weights = a.on.weights + s * a.on.weights_sequence + head * a.on.weights_head;
  int32_t* to_positions = a.to.positions + s * a.to.positions_sequence + head * a.to.positions_head;
  float* to_weights = a.to.weights + s * a.to.weights_sequence + head * a.to.weights_head;
  if (MOVES && head == 0 && thread == 0) a.to.lengths[s] = min(held, a.keep);
  if (held <= a.keep || a.keep == 0) {
    if (!MOVES && thread == 0) a.count[blockIdx.x] = 0;
    for (int t = thread; t < held && t < a.keep; t += kThreads) {
      if (to_positions != positions) to_positions[t] = positions[t];
      if (to_weights != weights) to_weights[t] = weights[t];
    }
    return;
  }

  // What stays where it is comes to its new place at once.  (After this no place is both read and written: what moves comes from `keep` on.)
  if (thread == 0) sh.newest = INT32_MIN;
  const int rows = (held + 255) / 256;  // pieces of 256 places
  constexpr int TURNS = PLACES / (kThreads * 4);
  int newest = INT32_MIN;
  int32_t p[TURNS][4];
  float w[TURNS][4];
  // (all loads are made, and none waits for another: behind what is held those of its last four places, since there is room for `capacity`, a multiple of 16)
#pragma unroll
  for (int i = 0; i < TURNS; ++i) {
    const int t = min((i * kThreads + thread) * 4, (held - 1) / 4 * 4);
    four(positions + t, p[i]);
    four(weights + t, w[i]);
  }
#pragma unroll
  for (int i = 0; i < TURNS; ++i) {
    const int t = (i * kThreads + thread) * 4;
    unsigned k[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      k[j] = t + j < held ? key_of(w[i][j]) : 0u;
      if (t + j < held) newest = max(newest, p[i][j]);
      if (t + j < a.keep && to_positions != positions) to_positions[t + j] = p[i][j];
      if (t + j < a.keep && to_weights != weights) to_weights[t + j] = w[i][j];
    }
    if (t < rows * 256) keys[t / 4] = uint4{k[0], k[1], k[2], k[3]};
  }
  if (a.recent) {
    for (int d = 32; d; d /= 2) newest = max(newest, __shfl_xor(newest, d));
    __syncthreads();
    if (lane == 0) atomicMax(&sh.newest, newest);
    __syncthreads();
    const int64_t oldest = (int64_t)sh.newest - a.recent;
#pragma unroll
    for (int i = 0; i < TURNS; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = (i * kThreads + thread) * 4 + j;
        if (t < held && p[i][j] > oldest) reinterpret_cast<unsigned*>(keys)[t] = kStays;
      }
  }
  const auto [prefix, left, equal] = choice(a.keep, sh, [&](auto show) {
    for (int i = thread; i < rows * 64; i += kThreads) {
      const uint4 k = keys[i];
      show(k.x), show(k.y), show(k.z), show(k.w);
    }
  });

  // Places that `is` picks, in their order: done(rank, place) for each.  Ranks within 256 places come from the lanes' votes.
  auto ranked = [&](auto is, auto done) {
    __syncthreads();
    for (int row = wave; row < rows; row += kWaves) {
      const uint4 k4 = keys[row * 64 + lane];
      const unsigned k[4] = {k4.x, k4.y, k4.z, k4.w};
      int n = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) n += __popcll(__ballot(is(k[j], row * 256 + lane * 4 + j)));
      if (lane == 0) counts[row] = n;
    }
    __syncthreads();
    if (wave == 0) {
      unsigned base = 0;
      for (int i = 0; i < rows; i += 64) {
        const unsigned v = i + lane < rows ? counts[i + lane] : 0;
        const unsigned sum = upto_lane(v);
        if (i + lane < rows) counts[i + lane] = base + sum - v;
        base += (unsigned)__builtin_amdgcn_readlane((int)sum, 63);
      }
      if (lane == 0) sh.total = base;
    }
    __syncthreads();
    for (int row = wave; row < rows; row += kWaves) {
      const uint4 k4 = keys[row * 64 + lane];
      const unsigned k[4] = {k4.x, k4.y, k4.z, k4.w};
      unsigned rank = counts[row];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const unsigned long long votes = __ballot(is(k[j], row * 256 + lane * 4 + j));
        rank = __builtin_amdgcn_mbcnt_hi((unsigned)(votes >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)votes, rank));
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (is(k[j], row * 256 + lane * 4 + j)) done(rank++, row * 256 + lane * 4 + j);
    }
  };

  if (equal != left)  // some of the ties go: the higher places, with a key that is one less (no key is 1, so that this is none's and not 0)
    ranked([&](unsigned k, int) { return k == prefix; }, [&](unsigned rank, int t) {
      if (rank >= left) reinterpret_cast<unsigned*>(keys)[t] = prefix - 1;
    });
  // places below `keep` that go and places from `keep` on that stay: as many of the one as of the other, and in this order
  __shared__ int32_t few[2 * kFew];
  int32_t* from = MOVES ? few : a.from + (int64_t)blockIdx.x * a.most;
  int32_t* into = MOVES ? few + kFew : a.into + (int64_t)blockIdx.x * a.most;
  ranked([&](unsigned k, int t) { return k && (k >= prefix) != (t < a.keep); }, [&](unsigned rank, int t) {
    if (t < a.keep) into[rank] = t;
    else from[rank - sh.total / 2] = t;
  });
  const int count = (int)(sh.total / 2);
  if (!MOVES && thread == 0) a.count[blockIdx.x] = count;
  __syncthreads();
  for (int i = thread; i < count; i += kThreads) {
    const int f = from[i], t = into[i];
    to_positions[t] = positions[f];
    to_weights[t] = weights[f];
  }
  if constexpr (MOVES)
    for (int i = thread / a.lanes; i < count; i += kThreads / a.lanes) move<1>(a, s, head, {from[i]}, {into[i]}, thread % a.lanes);
}

// The same for more places than LDS holds the keys of: these are formed again for every look at them, and a thread has a run of places.
__global__ void __launch_bounds__(kThreads) kv4_choose_long_kernel(Evict a) {
  __shared__ Shared sh;
  const int s = blockIdx.x / a.heads, head = blockIdx.x - s * a.heads_count;
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
  if (threadIdx.x == 0) sh.newest = newest;
  for (int t = threadIdx.x; t < held; t += kThreads) newest = max(newest, positions[t]);
  for (int d = 32; d; d /= 2) newest = max(newest, __shfl_xor(newest, d));
  __syncthreads();
  if (threadIdx.x % 64 == 0) atomicMax(&sh.newest, newest);
  __syncthreads();
  newest = sh.newest;

  const Choice c = choice(a.keep, sh, [&](auto show) {
    for (int t = threadIdx.x; t < held; t += kThreads) show(key_of(weights[t], positions[t], newest, a.recent));
  });
  const unsigned prefix = c.prefix, left = c.left;

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

__global__ void __launch_bounds__(256) kv4_move_kernel(Evict a) {
  const int s = blockIdx.x / a.heads, head = blockIdx.x - s * a.heads_count;
  if (blockIdx.y == 0 && head == 0 && threadIdx.x == 0) a.to.lengths[s] = min(kv_held(a.on.lengths, s, a.capacity), a.keep);
  const int count = a.count[blockIdx.x], per = 256 / a.lanes;
  const int32_t* from = a.from + (int64_t)blockIdx.x * a.most;
  const int32_t* into = a.into + (int64_t)blockIdx.x * a.most;
  for (int first = blockIdx.y * per + threadIdx.x / a.lanes; first < count; first += kAtOnce * gridDim.y * per) {
    int f[kAtOnce], t[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const int i = first + j * gridDim.y * per;
      f[j] = i < count ? from[i] : -1;
      t[j] = i < count ? into[i] : 0;
    }
    move<kAtOnce>(a, s, head, f, t, threadIdx.x % a.lanes);
  }
}

template <int PLACES>
hipError_t choose(const Evict& a, unsigned all, bool moves, hipStream_t st) {
  if (moves) hipLaunchKernelGGL((kv4_choose_kernel<PLACES, true>), dim3(all), dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((kv4_choose_kernel<PLACES, false>), dim3(all), dim3(kThreads), 0, st, a);
  return hipGetLastError();
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
  Evict a = {cache, on, to, (int)capacity, (int)(keep < capacity ? keep : capacity), (int)(recent < capacity ? recent : capacity), (int)most,
             (int)cache.page_size, (int)cache.heads, 1, fast_div((unsigned)cache.page_size), fast_div((unsigned)cache.heads), count, from, from + all * most};
  while (a.lanes * 8 < cache.dim) a.lanes *= 2;
  // Few moves are made by the workgroup that chose them, which saves a launch.  Not in place: others read the lengths while it would write them.
  const bool moves = most <= kFew && to.lengths != on.lengths && capacity <= 32768;
  hipError_t rc;
  if (capacity <= 8192) rc = choose<8192>(a, (unsigned)all, moves, st);
  else if (capacity <= 32768) rc = choose<32768>(a, (unsigned)all, moves, st);
  else {
    hipLaunchKernelGGL(kv4_choose_long_kernel, dim3((unsigned)all), dim3(kThreads), 0, st, a);
    rc = hipGetLastError();
  }
  if (rc != hipSuccess || moves) return rc;
  const int64_t blocks = (most * a.lanes + 256 * kAtOnce - 1) / (256 * kAtOnce);
  hipLaunchKernelGGL(kv4_move_kernel, dim3((unsigned)all, (unsigned)(blocks < 1 ? 1 : blocks < 256 ? blocks : 256)), dim3(256), 0, st, a);
  return hipGetLastError();
}
