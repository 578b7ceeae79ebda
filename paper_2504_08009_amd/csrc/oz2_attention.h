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
};

inline int64_t attention_tiles(const Attention& a, int64_t size) { return a.tokens * a.group / size + a.sequences; }

struct AttentionTile {
  int64_t begin;      // the sequence's first token
  int tokens, first;  // of the sequence, and the tile's first row
};
__device__ __forceinline__ AttentionTile attention_tile(const Attention& a, int64_t tile, int size) {
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
