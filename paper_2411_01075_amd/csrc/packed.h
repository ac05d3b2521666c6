// Attention over packed samples: what its entry points, its bf16 and its fp32 kernels share.
#pragma once
#include "kernels.h"

namespace cephalo {

// One entry of the work list that cephalo_packed_plan writes: 128 rows of a sample.
constexpr int kPackedTile = 128;
struct PackedTile { int first, rows, tile, spare; };      // the sample's first row, its rows, which 128 of them

// Samples one behind the other in the rows of qkv [tokens, ld]: heads * d columns of queries, kv_heads * d of keys, kv_heads * d of values.  Query head a
// reads key head a / group.
struct PackedArgs {
  const PackedTile* plan;
  int64_t tokens, ld, ldo;
  int tiles, heads, kv_heads, group, d;
  float scale;
};

// Which entry of the list and which of `units` heads a block works on.  The list has the longest work first, so the last blocks are short ones; the
// heads of an entry follow one another.  Blocks are dealt round-robin to the 8 XCDs, each with an L2 of its own: by_xcd gives each XCD an eighth
// of the heads, so that the heads that share keys (and the tiles of a head) find them in one L2.  Where an XCD would get half as much again as an
// equal share (5 heads, 12) the blocks go as they are dealt.
struct PackedOrder { int units, by_xcd; };
inline unsigned packed_grid(const PackedArgs& a, int units, PackedOrder* order) {
  const int64_t per = (units + 7) / 8;
  const bool by_xcd = 2 * 8 * per <= 3 * (int64_t)units;
  *order = {units, by_xcd};
  return (unsigned)(by_xcd ? 8 * per * a.tiles : (int64_t)units * a.tiles);
}
__device__ __forceinline__ bool packed_block(const PackedArgs& a, const PackedOrder& o, int l, PackedTile* t, int* unit) {
  int tile, u;
  if (o.by_xcd) {
    const int xcd = l & 7, i = l >> 3, per = (o.units + 7) >> 3, at = i % per;
    const int first = xcd * o.units >> 3, count = ((xcd + 1) * o.units >> 3) - first;
    if (at >= count) return false;
    tile = i / per; u = first + at;
  } else {
    tile = l / o.units; u = l % o.units;
  }
  // (the divisions run on the vector unit; readfirstlane tells the compiler that the results are uniform)
  tile = __builtin_amdgcn_readfirstlane(tile);
  *unit = __builtin_amdgcn_readfirstlane(u);
  const PackedTile e = a.plan[tile];
  *t = {__builtin_amdgcn_readfirstlane(e.first), __builtin_amdgcn_readfirstlane(e.rows), __builtin_amdgcn_readfirstlane(e.tile), 0};
  // (a list that is not this call's reaches no row outside the buffers)
  return t->first >= 0 && t->rows > 0 && t->tile >= 0 && (int64_t)t->first + t->rows <= a.tokens && (int64_t)t->tile * kPackedTile < t->rows;
}

int launch_attn_packed_fwd_mfma(const PackedArgs& a, int causal, const bf16* qkv, bf16* O, float* lse, hipStream_t s);
// dvec: [heads, tokens] fp32
int launch_attn_packed_bwd_mfma(const PackedArgs& a, int causal, const bf16* qkv, const bf16* O, const bf16* dO, const float* lse, float* dvec, bf16* dqkv, hipStream_t s);
int launch_attn_packed_fwd_f32(const PackedArgs& a, int causal, const float* qkv, float* O, float* lse, hipStream_t s);
int launch_attn_packed_bwd_f32(const PackedArgs& a, int causal, const float* qkv, const float* O, const float* dO, const float* lse, float* dvec, float* dqkv, hipStream_t s);

}  // namespace cephalo
