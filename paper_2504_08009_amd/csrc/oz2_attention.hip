// Attention over packed prompts (oz2_attention): which kernel a call takes.
#include "oz2_attention.h"

template <int XT> hipError_t oz2_attention_tile_of(const Attention& a, hipStream_t st);
extern template hipError_t oz2_attention_tile_of<OZ2_BF16>(const Attention&, hipStream_t);
extern template hipError_t oz2_attention_tile_of<OZ2_F16>(const Attention&, hipStream_t);

namespace {

// Rows whose pieces of eight values start at multiples of 16 bytes, and 64 of which lie within 2^31 bytes.
bool pieces(const oz2_rows& r, int64_t heads) {
  return (uintptr_t)r.data % 16 == 0 && r.ld_token % 8 == 0 && r.ld_token < (1 << 23) && (heads == 1 || r.ld_head % 8 == 0);
}
bool fours(const oz2_rows& r, int64_t heads) {
  return r.type == OZ2_F32 || ((uintptr_t)r.data % 8 == 0 && r.ld_token % 4 == 0 && (heads == 1 || r.ld_head % 4 == 0));
}

}  // namespace

hipError_t oz2_launch_attention(int64_t tokens, int64_t sequences, const int32_t* cu, int64_t heads, int64_t kv_heads, int64_t dim, float scale, int causal,
                                const oz2_rows& q, const oz2_rows& k, const oz2_rows& v, const oz2_rows& out, hipStream_t st) {
  Attention a = {cu, q, k, v, out, tokens, sequences, (int)heads, (int)kv_heads, (int)(heads / kv_heads), (int)dim, causal != 0,
                 scale * 1.44269504088896340736f, fast_div((unsigned)(heads / kv_heads)), out.type != OZ2_F32 && pieces(out, heads)};
  if (q.type != OZ2_F32 && dim % 8 == 0 && pieces(q, heads) && pieces(k, kv_heads) && pieces(v, kv_heads) && fours(out, heads))
    return q.type == OZ2_BF16 ? oz2_attention_tile_of<OZ2_BF16>(a, st) : oz2_attention_tile_of<OZ2_F16>(a, st);
  return oz2_attention_any(a, st);
}
