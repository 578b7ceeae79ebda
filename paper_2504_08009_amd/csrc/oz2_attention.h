// Attention over packed prompts (oz2_attention): how a call looks to its kernels, and how rows are shared out.
//
// The query heads of a kv head are rows beside each other: row r of a sequence is its token r / group, query head r % group, so that a tile of rows reads
// each key once for all of them.  Tiles of `size` rows are counted over all sequences without knowing their lengths on the host: sequence s has the tiles
// floor(cu[s] group / size) + s and on, which are at least as many as it needs.
#ifndef OZ2_ATTENTION_H
#define OZ2_ATTENTION_H

#include "oz2_kv4.h"
#include "oz2_fast_div.h"

#ifdef __HIPCC__

struct Attention {
  const int32_t* cu;
  oz2_rows q, k, v, out;
  int64_t tokens, sequences;
  int heads, kv_heads, group, dim, causal;
  float scale2;  // scale log2(e)
  FastDiv per_group;
  bool wide_out;  // the result's rows are 16-bit values in pieces of 16 bytes
};

inline int64_t attention_tiles(const Attention& a, int64_t size) { return a.tokens * a.group / size + a.sequences; }

struct AttentionTile {
  int64_t begin;      // the sequence's first token
  int tokens, first;  // of the sequence, and the tile's first row
};
__device__ __forceinline__ int attention_lanes_sum(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return __builtin_amdgcn_readlane(v, 63);
}
// The tile that is the `tile`-th to be worked on.  Up to 64 sequences: the tiles furthest from their sequences' begins come first, which with causal attention have
// the most to do, so that none of these is left to the end.  More: by sequences from the last on, each from its end.
__device__ __forceinline__ AttentionTile attention_tile(const Attention& a, int64_t tile, int64_t tiles, int size) {
  if (a.sequences <= 64) {
    const int lane = threadIdx.x % 64;
    int64_t begin = 0;
    int n = 0, own = 0;  // tokens and tiles of the lane's sequence
    if (lane < a.sequences) {
      const KvRange r = kv_range(a.cu, lane, a.tokens);
      begin = r.begin, n = (int)(r.end - r.begin);
      own = (int)(((int64_t)n * a.group + size - 1) / size);
    }
    // the largest number that more than `tile` tiles have before them in their sequence, or are at
    int low = 0, high = (int)tiles, behind = 0;  // count(low) > tile >= count(high) = behind
    if (attention_lanes_sum(own) <= tile) return {0, 0, 0};
    while (high - low > 1) {
      const int mid = low + (high - low) / 2, count = attention_lanes_sum(own > mid ? own - mid : 0);
      if (count > tile) low = mid;
      else high = mid, behind = count;
    }
    // of the sequences that have a tile `low`, the (tile - behind)-th
    unsigned long long left = __ballot(own > low);
    for (int64_t i = tile - behind; i > 0; --i) left &= left - 1;
    const int s = __builtin_amdgcn_readfirstlane(__ffsll((long long)left) - 1);
    const int64_t from = (int64_t)((uint64_t)(unsigned)__builtin_amdgcn_readlane((int)begin, s) | (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(begin >> 32), s) << 32);
    return {from, __builtin_amdgcn_readlane(n, s), low * size};
  }
  tile = tiles - 1 - tile;
  const int64_t low = kv_sequence(a.sequences, [&](int64_t i) {
    const int64_t cu = a.cu[i];
    return (cu < 0 ? 0 : cu) * a.group / size + i <= tile;
  });
  const KvRange r = kv_range(a.cu, low, a.tokens);
  const int64_t cu = a.cu[low], first = (tile - ((cu < 0 ? 0 : cu) * a.group / size + low)) * size;
  const int n = (int)(r.end - r.begin);
  // a tile that is none of the sequence's begins behind it
  return {r.begin, n, first < 0 || first >= (int64_t)n * a.group ? n * a.group : (int)first};
}

hipError_t oz2_attention_any(const Attention& a, hipStream_t st);

#endif
#endif
