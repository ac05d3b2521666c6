// bf16 attention over packed samples of different lengths with grouped heads, forward and backward, on the gfx950 matrix cores.
//
// Sample i is rows [start_i, start_i + S_i) of qkv; query head a reads key head g = a / group:
//   s = scale q k,  P = exp(s - lse),  O = P V;   dV_g = sum over the group's heads of P^T dO,  dS = P (dO V^T - rowsum(dO O)),
//   dQ = scale dS K,  dK_g = scale sum over the group's heads of dS^T Q.
// A block owns 128 rows of one sample (an entry of the work list) and one head: 128 queries and the keys they see in the forward and for dQ, 128 keys
// and the queries of all the group's heads that see them, one head after the other, for dK and dV, whose sums over the group are formed in the
// accumulators.  The buffers' descriptors cover one sample's rows: what a tile reaches past them arrives as zeros, so no sample meets another's values.
// Orientation of the products, tiles and fragments: attn_tile.h.
#include "attn_tile.h"
#include "packed.h"
#include "reserve_lds.h"

namespace cephalo {
namespace {

constexpr int kThreads8 = 512;

// one sample's rows of the packed projection, and of O or dO
struct SampleRows {
  const bf16* base;
  i32x4 rsrc;
  unsigned ld_bytes;
  __device__ __forceinline__ SampleRows(const bf16* m, int64_t ld, int first, int rows, int width) {
    base = m + (int64_t)first * ld;
    ld_bytes = (unsigned)ld * 2;
    rsrc = make_rsrc_words(base, (unsigned)(((int64_t)(rows - 1) * ld + width) * 2));
  }
};

template <int D> constexpr int kFwdWaves = D == 128 ? 2 : 4;
template <int D> constexpr int kDqWaves = D == 32 ? 4 : D == 64 ? 3 : 2;
template <int D> constexpr int kDkvWaves = D == 32 ? 3 : 2;

// ------------------------------------------------------------------------------------ forward
// Four wavefronts of 32 queries each, key tiles of 64 in two stages.  The queries of a wavefront see the tiles up to `mine`; it helps to stage the others.
template <int D, bool CAUSAL>
__global__ void __launch_bounds__(kThreads, kFwdWaves<D>)
packed_fwd_kernel(PackedArgs p, PackedOrder order, const bf16* __restrict__ qkv, bf16* __restrict__ O, float* __restrict__ lse) {
  typedef Tile<D> TL;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds_bf16* smem = (lds_bf16*)smem_raw;
  auto Ks = [&](int st) { return smem + st * 2 * TL::ELEMS; };
  auto Vs = [&](int st) { return smem + st * 2 * TL::ELEMS + TL::ELEMS; };
  PackedTile e;
  int a;
  if (!packed_tile(p, order, blockIdx.x, &e, &a)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
  const int S = e.rows, d = p.d, g = a / p.group;
  const SampleRows x(qkv, p.ld, e.first, S, (p.heads + 2 * p.kv_heads) * d);
  const unsigned k_bytes = (unsigned)((p.heads + g) * d * 2), v_bytes = k_bytes + (unsigned)(p.kv_heads * d * 2);
  const float c2 = p.scale * kLog2e;
  const int q0 = e.tile * 128 + wave * 32, q = q0 + (lane & 31);
  const int ntiles = ((CAUSAL ? min(S, e.tile * 128 + 128) : S) + TILE - 1) / TILE;

  bf16x8 qf[D / 16];
  load_row_frags<D>(x.base + a * d, p.ld, q0, S, qf, d);
  auto stage = [&](int kt) {
    if (kt >= ntiles) return;
    TL::stage(x.rsrc, k_bytes, x.ld_bytes, kt * TILE, Ks(kt & 1), d);
    TL::stage(x.rsrc, v_bytes, x.ld_bytes, kt * TILE, Vs(kt & 1), d);
  };
  auto close = [&] {
    __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0): this wavefront's rows have landed
    __syncthreads();
  };
  stage(0);
  close();

  FragAddr<D> at(smem);
  f32x16 o[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const int mine = q0 >= S ? 0 : CAUSAL ? min(ntiles, (q0 + 31) / TILE + 1) : ntiles;
  int kt = 0;
  for (; kt < mine; ++kt) {
    const int t0 = kt * TILE;
    stage(kt + 1);
    fwd_tile<D>(at, qf, o, m_run, l_run, c2, (CAUSAL && t0 + 63 > q0) || t0 + 64 > S, (CAUSAL ? min(q, S - 1) : S - 1) - t0 - 4 * h);
    at.flip();
    close();
  }
  for (; kt < ntiles; ++kt) {
    stage(kt + 1);
    close();
  }
  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  store_transposed<D>(o, O + (int64_t)e.first * p.ldo + a * d, p.ldo, q, S, 1.0f / l_tot, d);
  if (h == 0 && q < S) lse[(int64_t)a * p.tokens + e.first + q] = (m_run + __builtin_amdgcn_logf(l_tot)) * kLn2;
}

// ------------------------------------------------------------------------------------ dQ
template <int D, bool CAUSAL>
__global__ void __launch_bounds__(kThreads, kDqWaves<D>)
packed_dq_kernel(PackedArgs p, PackedOrder order, const bf16* __restrict__ qkv, const bf16* __restrict__ O, const bf16* __restrict__ dO,
                 const float* __restrict__ lse, float* __restrict__ dvec, bf16* __restrict__ dqkv) {
  typedef Tile<D> TL;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds_bf16* smem = (lds_bf16*)smem_raw;
  auto Ks = [&](int st) { return smem + st * 2 * TL::ELEMS; };
  auto Vs = [&](int st) { return smem + st * 2 * TL::ELEMS + TL::ELEMS; };
  PackedTile e;
  int a;
  if (!packed_tile(p, order, blockIdx.x, &e, &a)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
  const int S = e.rows, d = p.d, g = a / p.group;
  const SampleRows x(qkv, p.ld, e.first, S, (p.heads + 2 * p.kv_heads) * d);
  const unsigned k_bytes = (unsigned)((p.heads + g) * d * 2), v_bytes = k_bytes + (unsigned)(p.kv_heads * d * 2);
  const float c2 = p.scale * kLog2e;
  const int q0 = e.tile * 128 + wave * 32, q = q0 + (lane & 31);
  const int ntiles = ((CAUSAL ? min(S, e.tile * 128 + 128) : S) + TILE - 1) / TILE;

  bf16x8 qf[D / 16], dof[D / 16];
  const int64_t orow = (int64_t)e.first * p.ldo + a * d, stat = (int64_t)a * p.tokens + e.first + q;
  load_row_frags<D>(dO + orow, p.ldo, q0, S, dof, d);
  const float dv = row_dot<D>(O + orow, p.ldo, q0, S, dof, d);
  load_row_frags<D>(x.base + a * d, p.ld, q0, S, qf, d);
  const float lse2 = q < S ? lse[stat] * kLog2e : 0.f;
  if (h == 0 && q < S) dvec[stat] = dv;
  f32x16 dq[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) dq[dt][i] = 0.f;
  auto stage = [&](int kt) {
    if (kt >= ntiles) return;
    TL::stage(x.rsrc, k_bytes, x.ld_bytes, kt * TILE, Ks(kt & 1), d);
    TL::stage(x.rsrc, v_bytes, x.ld_bytes, kt * TILE, Vs(kt & 1), d);
  };
  auto close = [&] {
    __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0)
    __syncthreads();
  };
  stage(0);
  close();
  FragAddr<D> at(smem);
  const int mine = q0 >= S ? 0 : CAUSAL ? min(ntiles, (q0 + 31) / TILE + 1) : ntiles;
  int kt = 0;
  for (; kt < mine; ++kt) {
    const int t0 = kt * TILE;
    stage(kt + 1);
    dq_tile<D>(at, qf, dof, dq, c2, lse2, dv, (CAUSAL && t0 + 63 > q0) || t0 + 64 > S, (CAUSAL ? min(q, S - 1) : S - 1) - t0 - 4 * h);
    at.flip();
    close();
  }
  for (; kt < ntiles; ++kt) {
    stage(kt + 1);
    close();
  }
  store_transposed<D>(dq, dqkv + (int64_t)e.first * p.ld + a * d, p.ld, q, S, p.scale, d);
}

// The queries that a block of 128 keys walks: of each of the group's heads the tiles of 64 that see the keys, from step `begin` of that order on.
struct QueryWalk {
  int first, end, left, head, it;                      // tiles [first, end) of each head; steps left, the next step's head and tile
  __device__ __forceinline__ QueryWalk(const KeyItem& e, bool causal, int group) {
    first = walk_first(causal, e.tile) / TILE;
    end = (e.rows + TILE - 1) / TILE;
    const int per = end - first;
    left = e.end - e.begin;
    head = uniform(e.begin / per);
    it = first + e.begin - head * per;
  }
  __device__ __forceinline__ bool more() const { return left > 0; }
  __device__ __forceinline__ void step() {
    --left;
    if (++it == end) { it = first; ++head; }
  }
};
static_assert(kWalkRows == TILE, "a step of the walk is a tile");

// 16 values of each block of 32 columns (4 consecutive columns of one key, four times) to a place of the workspace, lanes next to one another
template <int D>
__device__ __forceinline__ void store_part(const f32x16 (&acc)[D / 32], float* part, int keys32) {
  f32x4* to = reinterpret_cast<f32x4*>(part) + (size_t)keys32 * (D / 8) * 64 + (threadIdx.x & 63);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) to[(dt * 4 + j) * 64] = f32x4{acc[dt][4 * j], acc[dt][4 * j + 1], acc[dt][4 * j + 2], acc[dt][4 * j + 3]};
}
// dV and dK of 32 keys: to their rows, or to the item's place
template <int D>
__device__ __forceinline__ void store_keys(const PackedArgs& p, const KeyItem& e, int g, int t, int keys32, const f32x16 (&dk)[D / 32], const f32x16 (&dvv)[D / 32], bf16* dqkv) {
  if (e.slot < 0) {
    bf16* out = dqkv + (int64_t)e.first * p.ld + (p.heads + g) * p.d;
    store_transposed<D>(dvv, out + p.kv_heads * p.d, p.ld, t, e.rows, 1.0f, p.d);
    store_transposed<D>(dk, out, p.ld, t, e.rows, p.scale, p.d);
  } else {
    float* part = p.part + ((size_t)e.slot * p.kv_heads + g) * (2 * kPackedTile * D);
    store_part<D>(dvv, part + kPackedTile * D, keys32);
    store_part<D>(dk, part, keys32);
  }
}
// The places of a join's pieces added in their order.  A thread has 4 columns of one key.
template <int D>
__global__ void __launch_bounds__(256) packed_join_kernel(PackedArgs p, bf16* __restrict__ dqkv) {
  const KeyItem e = p.joins[blockIdx.y];
  const int g = blockIdx.z, i = blockIdx.x * 256 + threadIdx.x, lane = i & 63, j = (i >> 6) % (D / 8), keys32 = i / (8 * D) % 4, which = i / (32 * D);
  const int t = e.tile * kPackedTile + keys32 * 32 + (lane & 31), d0 = 8 * j + 4 * (lane >> 5);
  if (!rows_fit(p, e.first, e.rows, e.tile) || t >= e.rows || d0 >= p.d || e.slot < 0 || e.slot + e.pieces > p.slots) return;
  const f32x4* part = reinterpret_cast<const f32x4*>(p.part) + ((size_t)e.slot * p.kv_heads + g) * (kPackedTile * D / 2) + i;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int q = 0; q < e.pieces; ++q) sum += part[(size_t)q * p.kv_heads * (kPackedTile * D / 2)];
  const float mul = which ? 1.0f : p.scale;
  bf16x4 v;
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = (bf16)(sum[k] * mul);
  *reinterpret_cast<bf16x4*>(dqkv + ((int64_t)e.first + t) * p.ld + (p.heads + which * p.kv_heads + g) * p.d + d0) = v;
}

// ------------------------------------------------------------------------------------ dK, dV, heads of 64 or less
// Four wavefronts of 32 keys, whose rows stay in registers.
template <int D, bool CAUSAL>
__global__ void __launch_bounds__(kThreads, kDkvWaves<D>)
packed_dkv_narrow_kernel(PackedArgs p, PackedOrder order, const bf16* __restrict__ qkv, const bf16* __restrict__ dO, const float* __restrict__ lse,
                         const float* __restrict__ dvec, bf16* __restrict__ dqkv) {
  typedef Tile<D> TL;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds_bf16* smem = (lds_bf16*)smem_raw;
  auto Qs = [&](int st) { return smem + st * 2 * TL::ELEMS; };
  auto dOs = [&](int st) { return smem + st * 2 * TL::ELEMS + TL::ELEMS; };
  LDS_AS float* stats = (LDS_AS float*)(smem + 4 * TL::ELEMS);      // [2 buffers][-lse / scale | -dvec][64]
  KeyItem e;
  int g;
  if (!packed_keys(p, order, blockIdx.x, CAUSAL, &e, &g)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
  const int S = e.rows, d = p.d, a0 = g * p.group;
  const SampleRows x(qkv, p.ld, e.first, S, (p.heads + 2 * p.kv_heads) * d), y(dO, p.ldo, e.first, S, p.heads * d);
  const float c2 = p.scale * kLog2e, per_scale = -1.0f / p.scale;
  const int t0 = e.tile * 128 + wave * 32, t = t0 + (lane & 31);

  QueryWalk next(e, CAUSAL, p.group), now = next;
  int buf = 0;                                         // where the next tile goes
  float rstat = 0.f;                                   // threads 0..63: of lse, 64..127: of dvec
  auto stage_next = [&] {
    if (!next.more()) return;
    const unsigned col = (unsigned)((a0 + next.head) * d * 2);
    TL::stage(x.rsrc, col, x.ld_bytes, next.it * TILE, Qs(buf), d);
    TL::stage(y.rsrc, col, y.ld_bytes, next.it * TILE, dOs(buf), d);
    rstat = 0.f;
    const int r = next.it * TILE + (threadIdx.x & 63);
    if (threadIdx.x < 128 && r < S) {
      const int64_t at = (int64_t)(a0 + next.head) * p.tokens + e.first + r;
      rstat = threadIdx.x < 64 ? lse[at] * per_scale : -dvec[at];
    }
  };
  auto close = [&] {                                   // the tile that was staged becomes the current one
    if (next.more()) {
      if (threadIdx.x < 128) stats[buf * 128 + threadIdx.x] = rstat;
      next.step();
      buf ^= 1;
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0)
    __syncthreads();
  };
  stage_next();
  bf16x8 kf[D / 16], vf[D / 16];
  load_row_frags<D>(x.base + (p.heads + g) * d, p.ld, t0, S, kf, d);
  load_row_frags<D>(x.base + (p.heads + p.kv_heads + g) * d, p.ld, t0, S, vf, d);
  f32x16 dk[D / 32], dvv[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) { dk[dt][i] = 0.f; dvv[dt][i] = 0.f; }
  FragAddr<D> at(smem);
  close();
  // of each head's tiles the wavefront's keys are seen from this one on; it helps to stage the others
  const int mine = t0 >= S ? now.end : CAUSAL ? max(now.first, t0 / TILE) : now.first;
  int cur = 0;
  while (now.more()) {
    for (; now.more() && now.it < mine; now.step()) {
      stage_next();
      at.flip();
      cur ^= 1;
      close();
    }
    for (; now.more() && now.it >= mine; now.step()) {
      stage_next();
      dkv_tile<D, CAUSAL, 64>(at, kf, vf, dk, dvv, stats + cur * 128 + 4 * h, c2, t0, t, now.it * TILE);
      at.flip();
      cur ^= 1;
      close();
    }
  }
  store_keys<D>(p, e, g, t, wave, dk, dvv, dqkv);
}

// ------------------------------------------------------------------------------------ dK, dV, heads of 65 to 128
// Eight wavefronts: wavefront w takes 32 of the 128 keys (w & 3) and of every 64 queries the 32 of half w >> 2.  The keys and values stay in LDS: in
// registers they would push the accumulators out of the file that the vector unit reads.
template <int D, bool CAUSAL>
__global__ void __launch_bounds__(kThreads8, 2)
packed_dkv_kernel(PackedArgs p, PackedOrder order, const bf16* __restrict__ qkv, const bf16* __restrict__ dO, const float* __restrict__ lse,
                  const float* __restrict__ dvec, bf16* __restrict__ dqkv) {
  typedef Tile<D, TILE, kThreads8> TL;
  typedef Tile<D, 128, kThreads8> TKV;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds_bf16* smem = (lds_bf16*)smem_raw;
  auto Qs = [&](int st) { return smem + st * 2 * TL::ELEMS; };
  auto dOs = [&](int st) { return smem + st * 2 * TL::ELEMS + TL::ELEMS; };
  lds_bf16* Ks = smem + 4 * TL::ELEMS;
  lds_bf16* Vs = Ks + TKV::ELEMS;
  LDS_AS float* stats = (LDS_AS float*)(Vs + TKV::ELEMS);   // [2 buffers][lse2 | dvec][64]
  KeyItem e;
  int g;
  if (!packed_keys(p, order, blockIdx.x, CAUSAL, &e, &g)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
  const int kg = wave & 3, qh = wave >> 2;
  const int S = e.rows, d = p.d, a0 = g * p.group;
  const SampleRows x(qkv, p.ld, e.first, S, (p.heads + 2 * p.kv_heads) * d), y(dO, p.ldo, e.first, S, p.heads * d);
  const float c2 = p.scale * kLog2e;
  const int t0 = e.tile * 128 + kg * 32, t = t0 + (lane & 31);

  const unsigned k_bytes = (unsigned)((p.heads + g) * d * 2), v_bytes = k_bytes + (unsigned)(p.kv_heads * d * 2);
  TKV::stage(x.rsrc, k_bytes, x.ld_bytes, e.tile * 128, Ks, d);
  TKV::stage(x.rsrc, v_bytes, x.ld_bytes, e.tile * 128, Vs, d);
  QueryWalk next(e, CAUSAL, p.group), now = next;
  int buf = 0;
  float rstat = 0.f;
  auto stage_next = [&] {
    if (!next.more()) return;
    const unsigned col = (unsigned)((a0 + next.head) * d * 2);
    TL::stage(x.rsrc, col, x.ld_bytes, next.it * TILE, Qs(buf), d);
    TL::stage(y.rsrc, col, y.ld_bytes, next.it * TILE, dOs(buf), d);
    rstat = 0.f;
    const int r = next.it * TILE + (threadIdx.x & 63);
    if (threadIdx.x < 128 && r < S) {
      const int64_t at = (int64_t)(a0 + next.head) * p.tokens + e.first + r;
      rstat = threadIdx.x < 64 ? lse[at] * kLog2e : dvec[at];
    }
  };
  auto close = [&] {
    if (next.more()) {
      if (threadIdx.x < 128) stats[buf * 128 + threadIdx.x] = rstat;
      next.step();
      buf ^= 1;
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0)
    __syncthreads();
  };
  stage_next();
  f32x16 dk[D / 32], dvv[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) { dk[dt][i] = 0.f; dvv[dt][i] = 0.f; }
  close();

  int cur = 0;
  for (; now.more(); now.step()) {
    stage_next();
    const LDS_AS float* st = stats + cur * 128;
    const int q0 = now.it * TILE + qh * 32;            // this wavefront's 32 queries
    if (CAUSAL ? q0 + 31 >= t0 : q0 < S && t0 < S) {
      constexpr int NP = D / 8;                        // products per phase
      f32x16 sc, dp;
#pragma unroll
      for (int i = 0; i < 16; ++i) { sc[i] = 0.f; dp[i] = 0.f; }
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(TL::frag_rows(Qs(cur), qh * 32, kk * 16), TKV::frag_rows(Ks, kg * 32, kk * 16), sc, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(TL::frag_rows(dOs(cur), qh * 32, kk * 16), TKV::frag_rows(Vs, kg * 32, kk * 16), dp, 0, 0, 0);
      }
      lds_ahead_schedule<NP, 2>();
      __builtin_amdgcn_sched_barrier(0);
      // P = exp2(S c2 - lse2) and dS = P (dP - dvec) as bf16 operands
      f32x16 pv, dsv;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = qh * 32 + 8 * j + 4 * h;         // 4 consecutive query rows
        const f32x4 l4 = *reinterpret_cast<const LDS_AS f32x4*>(st + r);
        const f32x4 d4 = *reinterpret_cast<const LDS_AS f32x4*>(st + 64 + r);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          pv[4 * j + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[4 * j + i], c2, -l4[i]));
          dsv[4 * j + i] = dp[4 * j + i] - d4[i];
        }
      }
      if ((CAUSAL && t0 + 31 > q0) || q0 + 32 > S) {    // diagonal or ragged end (wave-uniform)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int qq = q0 + 8 * (i >> 2) + 4 * h + (i & 3);
          if (qq >= S || (CAUSAL && t > qq)) pv[i] = 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) dsv[i] *= pv[i];
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) {
        const bf16x8 pf = pack8(pv, 8 * jj), df = pack8(dsv, 8 * jj);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
          dvv[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(TL::frag_cols(dOs(cur), dt * 32, qh * 32 + 16 * jj), pf, dvv[dt], 0, 0, 0);
          dk[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(TL::frag_cols(Qs(cur), dt * 32, qh * 32 + 16 * jj), df, dk[dt], 0, 0, 0);
        }
      }
      lds_ahead_schedule<NP, 2>();
    }
    cur ^= 1;
    close();
  }
  // the second half's sums go through LDS ([key group][value][lane], lanes contiguous) and the first half stores
  constexpr int NV = D / 32 * 16 * 2;
  LDS_AS float* mrg = (LDS_AS float*)smem_raw + kg * NV * 64 + lane;
  if (qh == 1) {
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        mrg[(dt * 16 + i) * 64] = dk[dt][i];
        mrg[(NV / 2 + dt * 16 + i) * 64] = dvv[dt][i];
      }
  }
  __syncthreads();
  if (qh == 0) {
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        dvv[dt][i] += mrg[(NV / 2 + dt * 16 + i) * 64];
        dk[dt][i] += mrg[(dt * 16 + i) * 64];
      }
    store_keys<D>(p, e, g, t, kg, dk, dvv, dqkv);
  }
}

template <int D, bool CAUSAL>
int fwd_cfg(const PackedArgs& a, const bf16* qkv, bf16* O, float* lse, hipStream_t s) {
  PackedOrder order;
  const unsigned grid = packed_grid(a.tiles, a.heads, &order);
  constexpr auto kern = packed_fwd_kernel<D, CAUSAL>;
  const size_t lds = 4 * (size_t)Tile<D>::ELEMS * sizeof(bf16);      // two stages of 64 keys and values
  if (const int rc = reserve_lds<kern>("attention_packed", lds); rc != CEPHALO_OK) return rc;
  kern<<<grid, kThreads, lds, s>>>(a, order, qkv, O, lse);
  CEPHALO_CHECK_LAUNCH("attention_packed_fwd");
  return CEPHALO_OK;
}

template <int D, bool CAUSAL>
int bwd_cfg(const PackedArgs& a, const bf16* qkv, const bf16* O, const bf16* dO, const float* lse, float* dvec, bf16* dqkv, hipStream_t s) {
  PackedOrder order;
  {
    const unsigned grid = packed_grid(a.tiles, a.heads, &order);
    constexpr auto kern = packed_dq_kernel<D, CAUSAL>;
    const size_t lds = 4 * (size_t)Tile<D>::ELEMS * sizeof(bf16);
    if (const int rc = reserve_lds<kern>("attention_packed", lds); rc != CEPHALO_OK) return rc;
    kern<<<grid, kThreads, lds, s>>>(a, order, qkv, O, dO, lse, dvec, dqkv);
    CEPHALO_CHECK_LAUNCH("attention_packed_dq");
  }
  const unsigned grid = packed_grid(a.key_items, a.kv_heads, &order);
  if constexpr (D <= 64) {
    constexpr auto kern = packed_dkv_narrow_kernel<D, CAUSAL>;
    const size_t lds = 4 * (size_t)Tile<D>::ELEMS * sizeof(bf16) + 2 * 128 * sizeof(float);
    if (const int rc = reserve_lds<kern>("attention_packed", lds); rc != CEPHALO_OK) return rc;
    kern<<<grid, kThreads, lds, s>>>(a, order, qkv, dO, lse, dvec, dqkv);
  } else {
    constexpr auto kern = packed_dkv_kernel<D, CAUSAL>;
    // staging (2 stages of Q and dO, the keys, the values, the row statistics) or, at the end, the merge of the halves
    const size_t staging = (4 * (size_t)Tile<D>::ELEMS + 2 * (size_t)Tile<D, 128>::ELEMS) * sizeof(bf16) + 2 * 128 * sizeof(float);
    const size_t merge = (size_t)4 * (D / 32 * 16 * 2) * 64 * sizeof(float);
    const size_t lds = staging > merge ? staging : merge;
    if (const int rc = reserve_lds<kern>("attention_packed", lds); rc != CEPHALO_OK) return rc;
    kern<<<grid, kThreads8, lds, s>>>(a, order, qkv, dO, lse, dvec, dqkv);
  }
  CEPHALO_CHECK_LAUNCH("attention_packed_dkv");
  if (a.join_items > 0) {
    packed_join_kernel<D><<<dim3(D / 4, a.join_items, a.kv_heads), 256, 0, s>>>(a, dqkv);
    CEPHALO_CHECK_LAUNCH("attention_packed_join");
  }
  return CEPHALO_OK;
}

}  // namespace

// a head that is not 32, 64 or 128 wide runs on the next of these tiles with the further columns held at zero
#define PACKED_FORMS(CALL)                                                              \
  if (a.d <= 32) return causal ? CALL(32, true) : CALL(32, false);                      \
  if (a.d <= 64) return causal ? CALL(64, true) : CALL(64, false);                      \
  return causal ? CALL(128, true) : CALL(128, false);

int launch_attn_packed_fwd_mfma(const PackedArgs& a, int causal, const bf16* qkv, bf16* O, float* lse, hipStream_t s) {
#define CALL(D, C) fwd_cfg<D, C>(a, qkv, O, lse, s)
  PACKED_FORMS(CALL)
#undef CALL
}
int launch_attn_packed_bwd_mfma(const PackedArgs& a, int causal, const bf16* qkv, const bf16* O, const bf16* dO, const float* lse, float* dvec, bf16* dqkv, hipStream_t s) {
#define CALL(D, C) bwd_cfg<D, C>(a, qkv, O, dO, lse, dvec, dqkv, s)
  PACKED_FORMS(CALL)
#undef CALL
}

}  // namespace cephalo
