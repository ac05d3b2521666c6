// C-ABI entry points of the operators on packed samples: the work list and the attention, rotary positions with several axes, dropout.
#include <algorithm>
#include <cmath>
#include "dropout.h"
#include "packed.h"
#include "positions.h"

using namespace cephalo;

namespace {
constexpr int64_t kRows = (int64_t)1 << 31;      // rows are counted in 32 bits
constexpr int kLongest = 1 << 30;                // of a sample, whose rows are added to and rounded up in them

int check_dtype(const char* who, int dtype) {
  if (dtype != CEPHALO_F32 && dtype != CEPHALO_BF16) return fail(CEPHALO_EINVAL, "%s: unknown dtype %d", who, dtype);
  return CEPHALO_OK;
}
int check_packed(const char* who, const cephalo_packed_desc* d) {
  if (!d) return fail(CEPHALO_EINVAL, "%s: null desc", who);
  if (d->heads <= 0 || d->heads > 65535 || d->kv_heads <= 0 || d->heads % d->kv_heads != 0)
    return fail(CEPHALO_EINVAL, "%s: %d query heads over %d key heads", who, d->heads, d->kv_heads);
  if (d->head_dim <= 0) return fail(CEPHALO_EINVAL, "%s: head dim %d must be positive", who, d->head_dim);
  if (d->head_dim > 128) return fail(CEPHALO_EUNSUPPORTED, "%s: head dim %d > 128", who, d->head_dim);
  if (const int rc = check_dtype(who, d->dtype); rc != CEPHALO_OK) return rc;
  const bool bf = d->dtype == CEPHALO_BF16;
  if (bf && d->head_dim % 8 != 0) return fail(CEPHALO_EUNSUPPORTED, "%s: bf16 needs a head dim that is a multiple of 8, got %d", who, d->head_dim);
  if (d->causal != 0 && d->causal != 1) return fail(CEPHALO_EINVAL, "%s: causal must be 0 or 1", who);
  // (the kernels hold scale * log2(e) and, of some heads, lse / scale in 32 bits)
  if (d->scale != 0.f && !(d->scale >= 1e-30f && d->scale <= 1e30f)) return fail(CEPHALO_EINVAL, "%s: scale %g must lie in 1e-30 to 1e30, or be 0 for 1/sqrt(head dim)", who, d->scale);
  if (d->tokens <= 0 || d->tokens >= kRows) return fail(CEPHALO_EINVAL, "%s: %lld rows", who, (long long)d->tokens);
  const int64_t o = (int64_t)d->heads * d->head_dim, qkv = o + 2 * (int64_t)d->kv_heads * d->head_dim;
  if (d->qkv_pitch < qkv || d->o_pitch < o)
    return fail(CEPHALO_EINVAL, "%s: pitches %lld and %lld do not cover rows of %lld and %lld", who, (long long)d->qkv_pitch, (long long)d->o_pitch, (long long)qkv, (long long)o);
  if (bf && (d->qkv_pitch % 8 != 0 || d->o_pitch % 8 != 0)) return fail(CEPHALO_EINVAL, "%s: bf16 rows must be 16-byte aligned: pitches %lld, %lld", who, (long long)d->qkv_pitch, (long long)d->o_pitch);
  if (d->qkv_pitch >= kRows || d->o_pitch >= kRows) return fail(CEPHALO_EUNSUPPORTED, "%s: pitches beyond 2^31", who);
  return CEPHALO_OK;
}
// a desc whose work list was made, and what the kernels' index arithmetic holds
int check_planned(const char* who, const cephalo_packed_desc* d) {
  if (const int rc = check_packed(who, d); rc != CEPHALO_OK) return rc;
  if (d->samples <= 0 || d->tiles < 0 || d->longest < 0 || d->longest > std::min<int64_t>(d->tokens, kLongest)) return fail(CEPHALO_EINVAL, "%s: cephalo_packed_plan has not filled this desc", who);
  if (d->dtype == CEPHALO_BF16 && ((int64_t)d->longest + kPackedTile) * std::max(d->qkv_pitch, d->o_pitch) * 2 >= kRows)
    return fail(CEPHALO_EUNSUPPORTED, "%s: a sample of %d rows exceeds the 2 GiB a buffer offset reaches", who, d->longest);
  if (d->key_items < d->tiles || d->joins < 0 || d->joins > d->tiles || d->slots < 0 || d->slots > d->key_items)
    return fail(CEPHALO_EINVAL, "%s: cephalo_packed_plan has not filled this desc", who);
  if (packed_threads(d->dtype == CEPHALO_F32, d->tiles, d->key_items, d->heads, d->kv_heads, d->head_dim) >= (int64_t)1 << 32)
    return fail(CEPHALO_EUNSUPPORTED, "%s: %d heads over %d tiles of 128 rows pass the 2^32 threads of a launch", who, d->heads, d->tiles);
  return CEPHALO_OK;
}
size_t part_bytes(const cephalo_packed_desc* d) { return (size_t)d->slots * d->kv_heads * packed_part_floats(d->head_dim) * sizeof(float); }
size_t dvec_bytes(const cephalo_packed_desc* d) { return ((size_t)d->heads * d->tokens * sizeof(float) + 255) / 256 * 256; }
PackedArgs packed_args(const cephalo_packed_desc* d, const void* plan) {
  PackedArgs a;
  a.plan = static_cast<const PackedTile*>(plan);
  a.keys = reinterpret_cast<const KeyItem*>(a.plan + d->tiles);
  a.joins = a.keys + d->key_items;
  a.key_items = d->key_items; a.join_items = d->joins; a.slots = d->slots;
  a.part = nullptr;
  a.tokens = d->tokens; a.ld = d->qkv_pitch; a.ldo = d->o_pitch;
  a.tiles = d->tiles; a.heads = d->heads; a.kv_heads = d->kv_heads; a.group = d->heads / d->kv_heads; a.d = d->head_dim;
  a.scale = d->scale > 0.f ? d->scale : 1.0f / std::sqrt((float)d->head_dim);
  return a;
}
bool all_aligned(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (!aligned16(p)) return false;
  return true;
}
}  // namespace

namespace {
// Pieces that a list cuts its keys' walks into, beyond one each: fewer than walk / share of each, and the share is at least all the steps over 512.
constexpr int kMostPieces = 512;

// How many steps of a walk an item takes, and by how many the longest walk may exceed that without any being cut.  A launch lasts as long as its longest block,
// and a key tile's walk is as long as the queries that see it times the heads that share it, so few keys and long walks leave the chip idle: walks
// are cut to an equal share of all steps on the blocks that run at once: 256 of eight wavefronts, twice that for heads up to 64 (fp32 cuts a tile's
// keys into eighths first).  Us of the whole backward without pieces, and with them: 2 x 512 tokens, 4 heads of 64 over 2, causal: 28 and 16; 700 + 300 + 100, 16 of 128 over 4: 96 and
// 33; 2048, 16 of 128 over 1: 1028 and 93; fp32, 2 x 512, 8 of 64 over 1: 222 and 83.
// Where the dQ blocks run in the same launch they fill what the longest items leave, so the share is 1.2 times as long (4096 tokens, 8 of 128 over 1: 152; 1.0 and
// 1.4 times: 162 and 168), and it is one of the blocks that they leave where that is a quarter or more (700 + 300 + 100: 33; never: 39).  Pieces pay for their places in the workspace
// and for the launch that joins them, as much as five steps (8 x 512, 8 of 64 over 8: 21; from none on 29; from twelve on, 2 x 512: 28 for 16), in fp32, whose steps take
// longer, two (2 x 197, 4 of 64 over 2: 23; five: 32); none is shorter than four steps (2 x 512: 16; eight: 20; fp32, 2 x 197, two: 31), and a walk is cut from 5/4 of a share on
// (700 + 300 + 100: 33; from 8/5 on: 41).
struct Share { int steps, slack; };
Share steps_an_item(const cephalo_packed_desc* d, int64_t tiles, int64_t steps) {
  const bool f32 = d->dtype == CEPHALO_F32, wide = d->head_dim > 64;
  const int64_t all = steps * d->kv_heads, blocks = f32 ? 32 : wide ? 256 : 512;
  double share = (double)all / blocks;
  if (!f32 && packed_one_launch(tiles, d->heads, d->kv_heads, d->head_dim)) {
    const int64_t left = blocks - tiles * d->heads * (wide ? 1 : 2);
    share *= 1.2;
    if (left >= blocks / 4) share = std::max(share, (double)all / left);
  }
  return {(int)std::min(std::max(std::ceil(share), 4.0), 1e9), f32 ? 2 : 5};
}
}  // namespace

extern "C" size_t cephalo_packed_plan_bytes(int32_t samples, int64_t tokens) {
  if (samples <= 0 || tokens < 0 || tokens >= kRows) return 0;
  const size_t tiles = (size_t)samples + (size_t)tokens / kPackedTile;
  return tiles * sizeof(PackedTile) + (2 * tiles + kMostPieces) * sizeof(KeyItem);
}

extern "C" int cephalo_packed_plan(cephalo_packed_desc* d, int32_t samples, const int32_t* starts, void* plan, size_t plan_bytes) {
  if (const int rc = check_packed("packed_plan", d); rc != CEPHALO_OK) return rc;
  if (samples <= 0) return fail(CEPHALO_EINVAL, "packed_plan: %d samples", samples);
  if (!starts || !plan) return fail(CEPHALO_EINVAL, "packed_plan: null buffer");
  if (plan_bytes < cephalo_packed_plan_bytes(samples, d->tokens))
    return fail(CEPHALO_EWORKSPACE, "packed_plan: %zu B < %zu B", plan_bytes, cephalo_packed_plan_bytes(samples, d->tokens));
  if (starts[0] < 0 || starts[samples] > d->tokens) return fail(CEPHALO_EINVAL, "packed_plan: samples from row %d to %d of %lld rows", starts[0], starts[samples], (long long)d->tokens);
  int longest = 0;
  for (int i = 0; i < samples; ++i) {
    if (starts[i + 1] < starts[i]) return fail(CEPHALO_EINVAL, "packed_plan: sample %d ends before it starts (rows %d, %d)", i, starts[i], starts[i + 1]);
    longest = std::max(longest, starts[i + 1] - starts[i]);
  }
  if (longest > kLongest) return fail(CEPHALO_EUNSUPPORTED, "packed_plan: a sample of %d rows, %d at most", longest, kLongest);
  PackedTile* list = static_cast<PackedTile*>(plan);
  const int causal = d->causal, group = d->heads / d->kv_heads;
  int tiles = 0;
  int64_t steps = 0, longest_walk = 0;
  for (int i = 0; i < samples; ++i) {
    const int rows = starts[i + 1] - starts[i];
    for (int t = 0; (int64_t)t * kPackedTile < rows; ++t) {
      list[tiles++] = {starts[i], rows, t, 0};
      const int64_t walk = (int64_t)walk_steps(causal, rows, t) * group;
      steps += walk;
      longest_walk = std::max(longest_walk, walk);
    }
  }
  std::sort(list, list + tiles, [causal](const PackedTile& a, const PackedTile& b) {
    const int wa = causal ? a.tile : a.rows, wb = causal ? b.tile : b.rows;
    return wa != wb ? wa > wb : a.first != b.first ? a.first < b.first : a.tile < b.tile;
  });
  // the walks, cut; an entry of the list stands for the keys of the same tile
  if (longest_walk > (int64_t)1 << 30) return fail(CEPHALO_EUNSUPPORTED, "packed_plan: %d rows under %d heads of a key head", longest, group);
  const Share share = steps_an_item(d, tiles, steps);
  const bool cut = longest_walk > (int64_t)share.steps + share.slack;
  int items = 0, joins = 0, slots = 0;
  KeyItem* keys = reinterpret_cast<KeyItem*>(list + tiles);
  for (int i = 0; i < tiles; ++i) {
    const PackedTile& e = list[i];
    const int64_t walk = (int64_t)walk_steps(causal, e.rows, e.tile) * group;
    const int pieces = cut && walk * 4 > (int64_t)share.steps * 5 ? (int)((walk + share.steps - 1) / share.steps) : 1;
    for (int q = 0; q < pieces; ++q)
      keys[items++] = {e.first, e.rows, e.tile, (int)(walk * q / pieces), (int)(walk * (q + 1) / pieces), pieces > 1 ? slots + q : -1, pieces, 0};
    if (pieces > 1) { slots += pieces; ++joins; }
  }
  KeyItem* join = keys + items;
  for (int i = 0, k = 0; i < items; ++i)
    if (keys[i].pieces > 1 && keys[i].begin == 0) join[k++] = keys[i];
  std::sort(keys, keys + items, [](const KeyItem& a, const KeyItem& b) {
    const int wa = a.end - a.begin, wb = b.end - b.begin;
    return wa != wb ? wa > wb : a.first != b.first ? a.first < b.first : a.tile != b.tile ? a.tile < b.tile : a.begin < b.begin;
  });
  d->samples = samples; d->longest = longest; d->tiles = tiles; d->key_items = items; d->joins = joins; d->slots = slots;
  d->plan_bytes = tiles * (int64_t)sizeof(PackedTile) + ((int64_t)items + joins) * (int64_t)sizeof(KeyItem);
  return CEPHALO_OK;
}

extern "C" int cephalo_op_attention_packed_fwd(const cephalo_packed_desc* d, const void* plan, const void* qkv, void* O, float* lse, void* stream) {
  if (const int rc = check_planned("attention_packed_fwd", d); rc != CEPHALO_OK) return rc;
  if (!plan || !qkv || !O || !lse) return fail(CEPHALO_EINVAL, "attention_packed_fwd: null buffer");
  if (!all_aligned({plan, qkv, O, lse})) return fail(CEPHALO_EINVAL, "attention_packed_fwd: buffers must be 16-byte aligned");
  if (d->tiles == 0) return CEPHALO_OK;
  const PackedArgs a = packed_args(d, plan);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (d->dtype == CEPHALO_F32) return launch_attn_packed_fwd_f32(a, d->causal, static_cast<const float*>(qkv), static_cast<float*>(O), lse, s);
  return launch_attn_packed_fwd_mfma(a, d->causal, static_cast<const bf16*>(qkv), static_cast<bf16*>(O), lse, s);
}

extern "C" size_t cephalo_op_attention_packed_bwd_workspace(const cephalo_packed_desc* d) {
  if (check_planned("attention_packed_bwd_workspace", d) != CEPHALO_OK) return 0;
  return dvec_bytes(d) + part_bytes(d);
}

extern "C" int cephalo_op_attention_packed_bwd(const cephalo_packed_desc* d, const void* plan, const void* qkv, const void* O, const void* dO,
                                               const float* lse, void* dqkv, void* workspace, size_t workspace_bytes, void* stream) {
  if (const int rc = check_planned("attention_packed_bwd", d); rc != CEPHALO_OK) return rc;
  if (!plan || !qkv || !O || !dO || !lse || !dqkv || !workspace) return fail(CEPHALO_EINVAL, "attention_packed_bwd: null buffer");
  if (!all_aligned({plan, qkv, O, dO, lse, dqkv, workspace})) return fail(CEPHALO_EINVAL, "attention_packed_bwd: buffers must be 16-byte aligned");
  if (workspace_bytes < cephalo_op_attention_packed_bwd_workspace(d))
    return fail(CEPHALO_EWORKSPACE, "attention_packed_bwd: workspace %zu B < %zu B", workspace_bytes, cephalo_op_attention_packed_bwd_workspace(d));
  if (d->tiles == 0) return CEPHALO_OK;
  PackedArgs a = packed_args(d, plan);
  float* dvec = static_cast<float*>(workspace);
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + dvec_bytes(d));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (d->dtype == CEPHALO_F32)
    return launch_attn_packed_bwd_f32(a, d->causal, static_cast<const float*>(qkv), static_cast<const float*>(O), static_cast<const float*>(dO), lse, dvec, static_cast<float*>(dqkv), s);
  return launch_attn_packed_bwd_mfma(a, d->causal, static_cast<const bf16*>(qkv), static_cast<const bf16*>(O), static_cast<const bf16*>(dO), lse, dvec, static_cast<bf16*>(dqkv), s);
}

extern "C" int cephalo_op_rotary_axes(int32_t dtype, const void* src, int64_t src_pitch, void* dst, int64_t dst_pitch, const int32_t* positions, int64_t rows,
                                      int32_t axes, const int32_t* axis_dims, int32_t heads, int32_t head_dim, double base, int32_t inverse, void* stream) {
  if (const int rc = check_dtype("rotary_axes", dtype); rc != CEPHALO_OK) return rc;
  const int vec = dtype == CEPHALO_F32 ? 4 : 8;
  if (rows < 0 || heads <= 0 || head_dim <= 0) return fail(CEPHALO_EINVAL, "rotary_axes: %lld rows of %d heads of %d", (long long)rows, heads, head_dim);
  if (head_dim > 2 * kMaxRotaryPairs || head_dim % vec != 0)
    return fail(CEPHALO_EUNSUPPORTED, "rotary_axes: head dim %d is not a multiple of %d up to %d", head_dim, vec, 2 * kMaxRotaryPairs);
  if (axes <= 0 || axes > kMaxAxes || !axis_dims) return fail(CEPHALO_EINVAL, "rotary_axes: %d axes, 1 to %d", axes, kMaxAxes);
  if (!(base > 1.0) || !std::isfinite(base)) return fail(CEPHALO_EINVAL, "rotary_axes: base %g must be above 1", base);
  if (inverse != 0 && inverse != 1) return fail(CEPHALO_EINVAL, "rotary_axes: inverse must be 0 or 1");
  const int64_t width = (int64_t)heads * head_dim;
  if (src_pitch < width || dst_pitch < width || src_pitch % vec != 0 || dst_pitch % vec != 0)
    return fail(CEPHALO_EINVAL, "rotary_axes: pitches %lld and %lld must cover %lld columns in multiples of %d", (long long)src_pitch, (long long)dst_pitch, (long long)width, vec);
  if (width >= kRows) return fail(CEPHALO_EUNSUPPORTED, "rotary_axes: rows of %lld columns", (long long)width);
  if (rows / rotary_split(heads, head_dim, vec).rows >= ((int64_t)1 << 32) / 256 - 1)
    return fail(CEPHALO_EUNSUPPORTED, "rotary_axes: %lld rows of %d heads pass the 2^32 threads of a launch", (long long)rows, heads);
  RotaryAxes r = {};
  r.src_pitch = src_pitch; r.dst_pitch = dst_pitch; r.heads = heads; r.d = head_dim; r.axes = axes;
  int pair = 0;
  for (int a = 0; a < axes; ++a) {
    if (axis_dims[a] < 0 || axis_dims[a] % 2 != 0 || axis_dims[a] > head_dim - 2 * pair)
      return fail(CEPHALO_EINVAL, "rotary_axes: axis %d turns %d columns: even widths, %d columns a head in all", a, axis_dims[a], head_dim);
    for (int i = 0; i < axis_dims[a] / 2; ++i, ++pair) {
      const double turns = std::pow(base, -2.0 * i / axis_dims[a]) / (2.0 * M_PI);
      r.turns[pair] = inverse ? -turns : turns;
      r.axis[pair] = (unsigned char)a;
    }
  }
  if (pair == 0) return fail(CEPHALO_EINVAL, "rotary_axes: no columns to turn");
  r.pairs = pair;
  if (rows == 0) return CEPHALO_OK;
  if (!src || !dst || !positions) return fail(CEPHALO_EINVAL, "rotary_axes: null buffer");
  if (!all_aligned({src, dst, positions})) return fail(CEPHALO_EINVAL, "rotary_axes: buffers must be 16-byte aligned");
  if (src == dst && src_pitch != dst_pitch) return fail(CEPHALO_EINVAL, "rotary_axes: in place, but pitches %lld and %lld", (long long)src_pitch, (long long)dst_pitch);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == CEPHALO_F32) return launch_rotary_axes<float>(r, static_cast<const float*>(src), static_cast<float*>(dst), positions, rows, s);
  return launch_rotary_axes<bf16>(r, static_cast<const bf16*>(src), static_cast<bf16*>(dst), positions, rows, s);
}

namespace {
int dropout_args(const char* who, int dtype, int64_t n, float p, uint64_t seed, int64_t first, const uint64_t* counter, DropoutArgs* d) {
  if (const int rc = check_dtype(who, dtype); rc != CEPHALO_OK) return rc;
  if (n < 0) return fail(CEPHALO_EINVAL, "%s: %lld elements", who, (long long)n);
  if (n >= kDropoutMost) return fail(CEPHALO_EUNSUPPORTED, "%s: %lld elements pass the 2^32 threads of a launch", who, (long long)n);
  if (!(p >= 0.f && p < 1.f)) return fail(CEPHALO_EINVAL, "%s: p %g is not in [0, 1)", who, p);
  const int drop = (int)std::floor((double)p * 65536.0 + 0.5);
  if (drop > 65535) return fail(CEPHALO_EINVAL, "%s: p %g leaves nothing", who, p);
  if (first < 0 || first % 8 != 0) return fail(CEPHALO_EINVAL, "%s: the first word %lld must be a multiple of 8", who, (long long)first);
  if (reinterpret_cast<uintptr_t>(counter) % 8 != 0) return fail(CEPHALO_EINVAL, "%s: the counter must be 8-byte aligned", who);
  *d = {n, seed, (uint64_t)first, counter, (unsigned)drop, (float)(65536.0 / (65536 - drop))};
  return CEPHALO_OK;
}
}  // namespace

extern "C" int cephalo_op_dropout_add(int32_t dtype, const void* branch, const float* resid, float* out, int64_t n, float p, uint64_t seed, int64_t first,
                                      const uint64_t* counter, void* stream) {
  DropoutArgs d;
  if (const int rc = dropout_args("dropout_add", dtype, n, p, seed, first, counter, &d); rc != CEPHALO_OK) return rc;
  if (n == 0) return CEPHALO_OK;
  if (!branch || !resid || !out) return fail(CEPHALO_EINVAL, "dropout_add: null buffer");
  if (!all_aligned({branch, resid, out})) return fail(CEPHALO_EINVAL, "dropout_add: buffers must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == CEPHALO_F32) return launch_dropout_add<float>(d, static_cast<const float*>(branch), resid, out, s);
  return launch_dropout_add<bf16>(d, static_cast<const bf16*>(branch), resid, out, s);
}

extern "C" int cephalo_op_dropout_bwd(int32_t dtype, const float* dy, void* dbranch, int64_t n, float p, uint64_t seed, int64_t first, const uint64_t* counter,
                                      void* stream) {
  DropoutArgs d;
  if (const int rc = dropout_args("dropout_bwd", dtype, n, p, seed, first, counter, &d); rc != CEPHALO_OK) return rc;
  if (n == 0) return CEPHALO_OK;
  if (!dy || !dbranch) return fail(CEPHALO_EINVAL, "dropout_bwd: null buffer");
  if (!all_aligned({dy, dbranch})) return fail(CEPHALO_EINVAL, "dropout_bwd: buffers must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == CEPHALO_F32) return launch_dropout_bwd<float>(d, dy, static_cast<float*>(dbranch), s);
  return launch_dropout_bwd<bf16>(d, dy, static_cast<bf16*>(dbranch), s);
}
