// fp32 attention over packed samples with grouped heads, forward and backward: the formulas and the blocks' shares of attn_packed.hip on the fp32 matrix
// products of attn_f32.hip.  A block owns 16 rows, an eighth of an entry of the work list, and its wavefronts take the blocks of 16 keys (queries) in
// turn, straight from memory; their results are merged in wavefront order.  Rows past a sample's end are read as zeros.
//
// What bounds it is the chain of loads and products of one block of 16, 3 to 5 us: eight wavefronts share it, or four where a head's registers
// allow no more, and the backward of heads up to 64 is one launch where few blocks run (dK / dV forms rowsum(dO O) itself).  611 tokens, the longest sample 401, 4 heads of 64 over 2,
// four wavefronts and two launches -> this: forward 23 -> 17 us, backward 53 -> 33 (with its join).
#include "attn_f32_tile.h"
#include "packed.h"

namespace cephalo {
namespace {

template <int P> constexpr int kW = packed_f32_waves(P);      // wavefronts of a block

// block l: an eighth of an entry (the eighths of an entry follow one another) and a head
__device__ __forceinline__ int packed_eighth(const PackedOrder& order, int l, int* place) {
  const int per = order.by_xcd ? 8 * ((order.units + 7) >> 3) : order.units;      // blocks of an entry in the order without eighths
  const int rest = l % (8 * per);
  *place = l / (8 * per) * per + rest % per;
  return uniform(rest / per);
}
__device__ __forceinline__ bool packed_queries(const PackedArgs& p, const PackedOrder& order, int l, PackedTile* e, int* head, int* row0) {
  int place;
  const int eighth = packed_eighth(order, l, &place);
  if (!packed_tile(p, order, place, e, head)) return false;
  *row0 = e->tile * kPackedTile + 16 * (7 - eighth);      // (the longest first)
  return *row0 < e->rows;
}

template <int P, bool VEC>
__global__ void __launch_bounds__(64 * kW<P>)
packed_f32_fwd_kernel(PackedArgs p, PackedOrder order, int causal, const float* __restrict__ qkv, float* __restrict__ O, float* __restrict__ lse) {
  const int block = blockIdx.x;
  __shared__ f32x4 red[(kW<P> - 1) * P * 64];
  __shared__ float ml[kW<P>][2][16];
  PackedTile e;
  int a, q0;
  if (!packed_queries(p, order, block, &e, &a, &q0)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
  const int S = e.rows, d = p.d, q = q0 + (lane & 15);
  const float* base = qkv + (int64_t)e.first * p.ld;
  const float* K = base + (int64_t)(p.heads + a / p.group) * d;
  const float* V = K + (int64_t)p.kv_heads * d;
  f32x4 qf[P], o[P];
  load_rows<P, VEC>(base + a * d, p.ld, q0, S, d, qf);
#pragma unroll
  for (int i = 0; i < P; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  const int end = causal ? min(S, q0 + 16) : S;
  for (int t0 = wave * 16; t0 < end; t0 += 16 * kW<P>) {
    f32x4 kf[P], vf[P];
    load_rows<P, VEC>(K, p.ld, t0, S, d, kf);
    load_cols<P>(V, p.ld, t0, S, d, vf);
    f32x4 s = dot_rows<P>(kf, qf);                         // scores of keys t0 + 4 g + i with query q
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = t0 + 4 * g + i;
      s[i] = (t < S && (!causal || t <= q)) ? s[i] * p.scale : -INFINITY;
      mx = fmaxf(mx, s[i]);
    }
    const float m_new = fmaxf(m, groups_max(mx));          // (this wavefront's maximum of the column)
    const float shift = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = expf(m - shift);
    f32x4 w;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) { w[i] = expf(s[i] - shift); sum += w[i]; }
    l = l * alpha + sum;
    m = m_new;
#pragma unroll
    for (int i = 0; i < P; ++i) o[i] *= alpha;
    if (causal && t0 == q0) add_weighted_diagonal<P>(o, vf, w, V, p.ld, t0, S, d, [&](int r) { return t0 + r > q; });
    else add_weighted<P>(o, vf, w);
  }
  l = groups_sum(l);
  if (g == 0) { ml[wave][0][lane] = m; ml[wave][1][lane] = l; }
  __syncthreads();
  float mx = -INFINITY, sum = 0.f;
#pragma unroll
  for (int w = 0; w < kW<P>; ++w) mx = fmaxf(mx, ml[w][0][lane & 15]);
  const float shift = mx == -INFINITY ? 0.f : mx;
#pragma unroll
  for (int w = 0; w < kW<P>; ++w) sum += ml[w][1][lane & 15] * expf(ml[w][0][lane & 15] - shift);
  const float mine = expf(m - shift);
#pragma unroll
  for (int i = 0; i < P; ++i) o[i] *= mine;
  merge_sums<P, kW<P>>(o, red);
  if (wave == 0) {
    store_columns<P>(O + (int64_t)e.first * p.ldo + a * d, p.ldo, q, S, d, o, 1.0f / sum);
    if (g == 0 && q < S) lse[(int64_t)a * p.tokens + e.first + q] = mx + logf(sum);
  }
}

// dvec: where rowsum(dO O) goes for the dK / dV blocks, or null
template <int P, bool VEC>
__device__ __forceinline__ void dq_block(const PackedArgs& p, const PackedOrder& order, int block, int causal, const float* __restrict__ qkv, const float* __restrict__ O,
                                         const float* __restrict__ dO, const float* __restrict__ lse, float* __restrict__ dvec, float* __restrict__ dqkv, f32x4* red) {
  PackedTile e;
  int a, q0;
  if (!packed_queries(p, order, block, &e, &a, &q0)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
  const int S = e.rows, d = p.d, q = q0 + (lane & 15);
  const float* base = qkv + (int64_t)e.first * p.ld;
  const float* K = base + (int64_t)(p.heads + a / p.group) * d;
  const float* V = K + (int64_t)p.kv_heads * d;
  const int64_t orow = (int64_t)e.first * p.ldo + a * d, stat = (int64_t)a * p.tokens + e.first;
  f32x4 qf[P], dof[P], dq[P];
  load_rows<P, VEC>(base + a * d, p.ld, q0, S, d, qf);
  load_rows<P, VEC>(dO + orow, p.ldo, q0, S, d, dof);
  const float dv = row_dot<P, VEC>(O + orow, p.ldo, q0, S, d, dof);
  if (dvec && wave == 0 && g == 0 && q < S) dvec[stat + q] = dv;
  const float l = lse[stat + min(q, S - 1)];
#pragma unroll
  for (int i = 0; i < P; ++i) dq[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int end = causal ? min(S, q0 + 16) : S;
  for (int t0 = wave * 16; t0 < end; t0 += 16 * kW<P>) {
    f32x4 kf[P], vf[P], kc[P];
    load_rows<P, VEC>(K, p.ld, t0, S, d, kf);
    load_rows<P, VEC>(V, p.ld, t0, S, d, vf);
    load_cols<P>(K, p.ld, t0, S, d, kc);
    const f32x4 s = dot_rows<P>(kf, qf), dp = dot_rows<P>(vf, dof);
    f32x4 dz;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = t0 + 4 * g + i;
      dz[i] = (t < S && (!causal || t <= q)) ? expf(s[i] * p.scale - l) * (dp[i] - dv) : 0.f;
    }
    if (causal && t0 == q0) add_weighted_diagonal<P>(dq, kc, dz, K, p.ld, t0, S, d, [&](int r) { return t0 + r > q; });
    else add_weighted<P>(dq, kc, dz);
  }
  merge_sums<P, kW<P>>(dq, red);
  if (wave == 0) store_columns<P>(dqkv + (int64_t)e.first * p.ld + a * d, p.ld, q, S, d, dq, p.scale);
}

// OWN: rowsum(dO O) is formed here, from O, not read from dvec
template <int P, bool VEC, bool OWN>
__device__ __forceinline__ void dkv_block(const PackedArgs& p, const PackedOrder& order, int block, int causal, const float* __restrict__ qkv, const float* __restrict__ O,
                                          const float* __restrict__ dO, const float* __restrict__ lse, const float* __restrict__ dvec, float* __restrict__ dqkv, f32x4* red) {
  KeyItem e;
  int kv, place;
  const int eighth = packed_eighth(order, block, &place);
  if (!packed_keys(p, order, place, causal, &e, &kv)) return;
  const int t0 = e.tile * kPackedTile + 16 * eighth;
  if (t0 >= e.rows) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
  const int S = e.rows, d = p.d, t = t0 + (lane & 15);
  const float* base = qkv + (int64_t)e.first * p.ld;
  const float* K = base + (int64_t)(p.heads + kv) * d;
  f32x4 kf[P], vf[P], dk[P], dvv[P];
  load_rows<P, VEC>(K, p.ld, t0, S, d, kf);
  load_rows<P, VEC>(K + (int64_t)p.kv_heads * d, p.ld, t0, S, d, vf);
#pragma unroll
  for (int i = 0; i < P; ++i) { dk[i] = f32x4{0.f, 0.f, 0.f, 0.f}; dvv[i] = f32x4{0.f, 0.f, 0.f, 0.f}; }
  const int per = walk_steps(causal, S, e.tile);
  // (four wavefronts share a step)
  for (int step = e.begin + (wave >> 2); step < e.end; step += kW<P> / 4) {
    const int a = kv * p.group + step / per, q0 = walk_first(causal, e.tile) + step % per * kWalkRows + (wave & 3) * 16;
    if (q0 >= S || (causal && q0 < t0)) continue;        // (16 rows that all lie before the keys see none of them)
    const float* Q = base + a * d;
    const float* D = dO + (int64_t)e.first * p.ldo + a * d;
    const int64_t stat = (int64_t)a * p.tokens + e.first;
    f32x4 qf[P], dof[P], qc[P], doc[P];
    load_rows<P, VEC>(Q, p.ld, q0, S, d, qf);
    load_rows<P, VEC>(D, p.ldo, q0, S, d, dof);
    load_cols<P>(Q, p.ld, q0, S, d, qc);
    load_cols<P>(D, p.ldo, q0, S, d, doc);
    f32x4 l, dv;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int q = min(q0 + 4 * g + i, S - 1);
      l[i] = lse[stat + q];
      if (!OWN) dv[i] = dvec[stat + q];
    }
    if (OWN) {
      const float own = row_dot<P, VEC>(O + (int64_t)e.first * p.ldo + a * d, p.ldo, q0, S, d, dof);
#pragma unroll
      for (int i = 0; i < 4; ++i) dv[i] = __shfl(own, 4 * g + i, 64);
    }
    const f32x4 s = dot_rows<P>(qf, kf), dp = dot_rows<P>(dof, vf);      // rows: queries q0 + 4 g + i, column: key t
    f32x4 w, dz;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int q = q0 + 4 * g + i;
      const bool ok = q < S && (!causal || t <= q);
      w[i] = ok ? expf(s[i] * p.scale - l[i]) : 0.f;
      dz[i] = ok ? w[i] * (dp[i] - dv[i]) : 0.f;
    }
    if (causal && q0 == t0) {
      add_weighted_diagonal<P>(dvv, doc, w, D, p.ldo, q0, S, d, [&](int r) { return q0 + r < t; });
      add_weighted_diagonal<P>(dk, qc, dz, Q, p.ld, q0, S, d, [&](int r) { return q0 + r < t; });
    } else {
      add_weighted<P>(dvv, doc, w);
      add_weighted<P>(dk, qc, dz);
    }
  }
  float *to_k = dqkv + (int64_t)e.first * p.ld + (int64_t)(p.heads + kv) * d, *to_v = to_k + (int64_t)p.kv_heads * d;
  int64_t ld = p.ld;
  int row = t, rows = S;
  if (e.slot >= 0) {                                     // a place of the workspace: [dK | dV][128][packed_width]
    ld = packed_width(d);
    to_k = p.part + ((size_t)e.slot * p.kv_heads + kv) * (2 * kPackedTile * ld);
    to_v = to_k + kPackedTile * ld;
    row = t - e.tile * kPackedTile;
    rows = S - e.tile * kPackedTile;
  }
  merge_sums<P, kW<P>>(dvv, red);
  if (wave == 0) store_columns<P>(to_v, ld, row, rows, d, dvv, 1.0f);
  merge_sums<P, kW<P>>(dk, red);
  if (wave == 0) store_columns<P>(to_k, ld, row, rows, d, dk, e.slot >= 0 ? 1.0f : p.scale);
}

template <int P, bool VEC>
__global__ void __launch_bounds__(64 * kW<P>)
packed_f32_dq_kernel(PackedArgs p, PackedOrder order, int causal, const float* __restrict__ qkv, const float* __restrict__ O, const float* __restrict__ dO,
                     const float* __restrict__ lse, float* __restrict__ dvec, float* __restrict__ dqkv) {
  __shared__ f32x4 red[(kW<P> - 1) * P * 64];
  dq_block<P, VEC>(p, order, blockIdx.x, causal, qkv, O, dO, lse, dvec, dqkv, red);
}
template <int P, bool VEC>
__global__ void __launch_bounds__(64 * kW<P>)
packed_f32_dkv_kernel(PackedArgs p, PackedOrder order, int causal, const float* __restrict__ qkv, const float* __restrict__ dO, const float* __restrict__ lse,
                      const float* __restrict__ dvec, float* __restrict__ dqkv) {
  __shared__ f32x4 red[(kW<P> - 1) * P * 64];
  dkv_block<P, VEC, false>(p, order, blockIdx.x, causal, qkv, nullptr, dO, lse, dvec, dqkv, red);
}
template <int P, bool VEC>
__global__ void __launch_bounds__(64 * kW<P>)
packed_f32_bwd_kernel(PackedArgs p, PackedOrder by_keys, PackedOrder by_queries, int key_blocks, int causal, const float* __restrict__ qkv, const float* __restrict__ O,
                      const float* __restrict__ dO, const float* __restrict__ lse, float* __restrict__ dqkv) {
  __shared__ f32x4 red[(kW<P> - 1) * P * 64];
  const int block = blockIdx.x;
  if (block < key_blocks) dkv_block<P, VEC, true>(p, by_keys, block, causal, qkv, O, dO, lse, nullptr, dqkv, red);
  else dq_block<P, VEC>(p, by_queries, block - key_blocks, causal, qkv, O, dO, lse, nullptr, dqkv, red);
}

// The places of a join's pieces added in their order, one value a thread.
__global__ void __launch_bounds__(256) packed_f32_join_kernel(PackedArgs p, float* __restrict__ dqkv) {
  const KeyItem e = p.joins[blockIdx.y];
  const int g = blockIdx.z, width = packed_width(p.d), i = blockIdx.x * 256 + threadIdx.x, c = i % width, row = i / width % kPackedTile, which = i / (kPackedTile * width);
  const int t = e.tile * kPackedTile + row;
  if (!rows_fit(p, e.first, e.rows, e.tile) || t >= e.rows || c >= p.d || e.slot < 0 || e.pieces > p.slots - e.slot) return;
  const size_t place = 2 * (size_t)kPackedTile * width;
  const float* part = p.part + ((size_t)e.slot * p.kv_heads + g) * place + i;
  float sum = 0.f;
  for (int q = 0; q < e.pieces; ++q) sum += part[(size_t)q * p.kv_heads * place];
  dqkv[((int64_t)e.first + t) * p.ld + (int64_t)(p.heads + which * p.kv_heads + g) * p.d + c] = sum * (which ? 1.0f : p.scale);
}

// pieces of 16 dimensions: 2, 4, 6 or 8 (a head in between runs on the next with zeros)
#define PACKED_F32_PIECES(CALL, VEC) \
  if (pieces <= 2) { CALL(2, VEC) } else if (pieces <= 4) { CALL(4, VEC) } else if (pieces <= 6) { CALL(6, VEC) } else { CALL(8, VEC) }
#define PACKED_F32_FORMS(CALL)              \
  const int pieces = (a.d + 15) / 16;       \
  if (vec) { PACKED_F32_PIECES(CALL, true) } else { PACKED_F32_PIECES(CALL, false) }
}  // namespace

int launch_attn_packed_fwd_f32(const PackedArgs& a, int causal, const float* qkv, float* O, float* lse, hipStream_t s) {
  const bool vec = a.d % 4 == 0 && a.ld % 4 == 0;
  PackedOrder order;
  const unsigned grid = 8 * packed_grid(a.tiles, a.heads, &order);
#define CALL(P, V) packed_f32_fwd_kernel<P, V><<<grid, 64 * kW<P>, 0, s>>>(a, order, causal, qkv, O, lse);
  PACKED_F32_FORMS(CALL)
#undef CALL
  CEPHALO_CHECK_LAUNCH("attention_packed_fwd");
  return CEPHALO_OK;
}

int launch_attn_packed_bwd_f32(const PackedArgs& a, int causal, const float* qkv, const float* O, const float* dO, const float* lse, float* dvec, float* dqkv, hipStream_t s) {
  const bool vec = a.d % 4 == 0 && a.ld % 4 == 0 && a.ldo % 4 == 0;
  PackedOrder order, by_keys;
  const unsigned grid = 8 * packed_grid(a.tiles, a.heads, &order), key_grid = 8 * packed_grid(a.key_items, a.kv_heads, &by_keys);
  // One launch, us in two and in one, by blocks: 448: 39 and 27; 864: 93 and 84; 1376: 248 and 226; 1536: 95 and 100; 4096: 434 and 459.  (Wider heads: the two
  // halves together spill.)
  if ((int64_t)grid + key_grid <= 1408 && a.d <= 64) {
#define CALL(P, V) packed_f32_bwd_kernel<P, V><<<grid + key_grid, 64 * kW<P>, 0, s>>>(a, by_keys, order, (int)key_grid, causal, qkv, O, dO, lse, dqkv);
    if (vec) { if (a.d <= 32) { CALL(2, true) } else { CALL(4, true) } }
    else { if (a.d <= 32) { CALL(2, false) } else { CALL(4, false) } }
#undef CALL
  } else {
#define CALL(P, V)                                                                                                       \
  packed_f32_dq_kernel<P, V><<<grid, 64 * kW<P>, 0, s>>>(a, order, causal, qkv, O, dO, lse, dvec, dqkv);                 \
  CEPHALO_CHECK_LAUNCH("attention_packed_dq");                                                                           \
  packed_f32_dkv_kernel<P, V><<<key_grid, 64 * kW<P>, 0, s>>>(a, by_keys, causal, qkv, dO, lse, dvec, dqkv);
    PACKED_F32_FORMS(CALL)
#undef CALL
  }
  CEPHALO_CHECK_LAUNCH("attention_packed_bwd");
  if (a.join_items > 0) {
    packed_f32_join_kernel<<<dim3(packed_width(a.d), a.join_items, a.kv_heads), 256, 0, s>>>(a, dqkv);
    CEPHALO_CHECK_LAUNCH("attention_packed_join");
  }
  return CEPHALO_OK;
}

}  // namespace cephalo
