// Attention over packed samples: what its entry points, its bf16 and its fp32 kernels share.
#pragma once
#include "kernels.h"

namespace cephalo {

// The work list that cephalo_packed_plan writes: `tiles` PackedTiles, then `key_items` KeyItems, then `joins` KeyItems.
constexpr int kPackedTile = 128;
struct PackedTile { int first, rows, tile, spare; };      // 128 rows of a sample: its first row, its rows, which 128 of them
// 128 keys of a sample and some of the queries that see them, for dK and dV.  The queries of the heads that share the keys, one head after the other, in
// steps of kWalkRows rows from the first that sees a key: steps [begin, end).  Where an item has them all it writes the results
// (slot -1), otherwise its 32-bit sums go to place `slot` of the workspace and the join of the same keys adds the `pieces` places from `slot` on.
struct KeyItem { int first, rows, tile, begin, end, slot, pieces, spare; };
constexpr int kWalkRows = 64;

// Samples one behind the other in the rows of qkv [tokens, ld]: heads * d columns of queries, kv_heads * d of keys, kv_heads * d of values.  Query head a
// reads key head a / group.
struct PackedArgs {
  const PackedTile* plan;
  const KeyItem* keys;
  const KeyItem* joins;
  int64_t tokens, ld, ldo;
  int tiles, key_items, join_items, slots, heads, kv_heads, group, d;
  float scale;
  float* part;             // dK and dV sums of the items that have a slot: [slot][kv head][packed_part_floats]
};
__host__ __device__ inline int packed_width(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }      // the tile a head of d columns runs on
inline size_t packed_part_floats(int d) { return 2 * (size_t)kPackedTile * packed_width(d); }

// Whether the bf16 backward is one launch: where its two halves, one after the other, would leave compute units idle.  Us in two and in one, by tiles times
// (heads + key heads).  Heads of 64: 768: 54 and 48; 864: 78 and 70; 1024: 34 and 34 (16 x 197), 229 and 217 (4096); 1216: 68 and 67; 1280: 76 and 73 (8 x 512), 163 and 175
// (2 x 2048); 1536: 112 and 117, 48 and 49; 1920: 137 and 142.  Heads of 32: 512: 22 and 16; 768: 33 and 30; 1280: 46 and 50; 1536: 74 and 81.  Heads of 65 to 128: 512: 44
// and 40; 640: 82 and 75, 175 and 163; 760: 88 and 86; 768: 45 and 55 (16 x 197, 104 columns); 1024: 90 and 106.  (Two: dQ blocks of 128 queries.)
inline bool packed_one_launch(int64_t tiles, int heads, int kv_heads, int d) { return tiles * (heads + kv_heads) <= (d <= 64 ? 1024 : 640); }

// Steps of a tile's keys over all the heads that share them, and the first row that sees one.
__host__ __device__ inline int walk_first(int causal, int tile) { return causal ? tile * kPackedTile : 0; }
__host__ __device__ inline int walk_steps(int causal, int rows, int tile) { return (rows - walk_first(causal, tile) + kWalkRows - 1) / kWalkRows; }

// Which entry of the list and which of `units` heads a block works on.  The list has the longest work first, so the last blocks are short ones; the
// heads of an entry follow one another.  Blocks are dealt round-robin to the 8 XCDs, each with an L2 of its own: by_xcd gives each XCD an eighth
// of the heads, so that the heads that share keys (and the tiles of a head) find them in one L2.  Where an XCD would get half as much again as an
// equal share (5 heads, 12) the blocks go as they are dealt.
struct PackedOrder { int units, by_xcd; };
inline int64_t packed_blocks(int entries, int units, PackedOrder* order) {
  const int64_t per = (units + 7) / 8;
  const bool by_xcd = 2 * 8 * per <= 3 * (int64_t)units;
  *order = {units, by_xcd};
  return by_xcd ? 8 * per * entries : (int64_t)units * entries;
}
inline unsigned packed_grid(int entries, int units, PackedOrder* order) { return (unsigned)packed_blocks(entries, units, order); }
// Wavefronts of an fp32 block, by its head's pieces of 16 columns; an fp32 block has an eighth of an entry's rows.
constexpr int packed_f32_waves(int pieces) { return pieces <= 6 ? 8 : 4; }
// The threads of the largest launch (of its first dimension) that a call makes: a launch takes fewer than 2^32.
inline int64_t packed_threads(int f32, int tiles, int key_items, int heads, int kv_heads, int d) {
  PackedOrder order;
  const int64_t queries = packed_blocks(tiles, heads, &order), keys = packed_blocks(key_items, kv_heads, &order);
  if (f32) return (queries > keys ? queries : keys) * 8 * 64 * packed_f32_waves((d + 15) / 16);
  const int64_t by_queries = queries * 256, by_keys = keys * (d <= 64 ? 256 : 512);
  return by_queries > by_keys ? by_queries : by_keys;
}
__device__ __forceinline__ bool packed_block(const PackedOrder& o, int l, int* entry, int* unit) {
  int e, u;
  bool any = true;
  if (o.by_xcd) {
    const int xcd = l & 7, i = l >> 3, per = (o.units + 7) >> 3, at = i % per;
    const int first = xcd * o.units >> 3, count = ((xcd + 1) * o.units >> 3) - first;
    any = at < count;
    e = i / per; u = first + at;
  } else {
    e = l / o.units; u = l % o.units;
  }
  // (the divisions run on the vector unit; readfirstlane tells the compiler that the results are uniform)
  *entry = __builtin_amdgcn_readfirstlane(e);
  *unit = __builtin_amdgcn_readfirstlane(u);
  return any;
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
// (a list that is not this call's reaches no row outside the buffers)
__device__ __forceinline__ bool rows_fit(const PackedArgs& a, int first, int rows, int tile) {
  return first >= 0 && rows > 0 && tile >= 0 && (int64_t)first + rows <= a.tokens && (int64_t)tile * kPackedTile < rows;
}
__device__ __forceinline__ bool packed_tile(const PackedArgs& a, const PackedOrder& o, int l, PackedTile* t, int* unit) {
  int entry;
  if (!packed_block(o, l, &entry, unit)) return false;
  const PackedTile e = a.plan[entry];
  *t = {uniform(e.first), uniform(e.rows), uniform(e.tile), 0};
  return rows_fit(a, t->first, t->rows, t->tile);
}
__device__ __forceinline__ bool packed_keys(const PackedArgs& a, const PackedOrder& o, int l, int causal, KeyItem* t, int* unit) {
  int entry;
  if (!packed_block(o, l, &entry, unit)) return false;
  const KeyItem e = a.keys[entry];
  *t = {uniform(e.first), uniform(e.rows), uniform(e.tile), uniform(e.begin), uniform(e.end), uniform(e.slot), uniform(e.pieces), 0};
  return rows_fit(a, t->first, t->rows, t->tile) && t->begin >= 0 && t->begin < t->end && t->slot < a.slots &&
         t->end <= walk_steps(causal, t->rows, t->tile) * a.group;
}

int launch_attn_packed_fwd_mfma(const PackedArgs& a, int causal, const bf16* qkv, bf16* O, float* lse, hipStream_t s);
// dvec: [heads, tokens] fp32
int launch_attn_packed_bwd_mfma(const PackedArgs& a, int causal, const bf16* qkv, const bf16* O, const bf16* dO, const float* lse, float* dvec, bf16* dqkv, hipStream_t s);
int launch_attn_packed_fwd_f32(const PackedArgs& a, int causal, const float* qkv, float* O, float* lse, hipStream_t s);
int launch_attn_packed_bwd_f32(const PackedArgs& a, int causal, const float* qkv, const float* O, const float* dO, const float* lse, float* dvec, float* dqkv, hipStream_t s);

}  // namespace cephalo
