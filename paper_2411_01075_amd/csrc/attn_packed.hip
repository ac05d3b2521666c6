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

template <int D> constexpr int kFwdWaves = D == 128 ? 2 : 3;
template <int D> constexpr int kDqWaves = D == 32 ? 4 : D == 64 ? 3 : 2;
template <int D> constexpr int kDkvWaves = D == 32 ? 3 : 2;

// ------------------------------------------------------------------------------------ forward
// What bounds it.  For heads of 128 a tile of 64 keys gives each wavefront 32 products of 32 x 32 x 16 (17 to 21 ns each, by the chip's power), one KiB of LDS
// for each, and 32 exponentials a lane.  LDS gives 128 bytes a clock to four SIMDs, just what the products take, and the tiles' arrival is a quarter more.
// A wavefront alone on its SIMD issues an instruction of the vector unit every 8 clocks, two together one every 4, so the exponentials have to run
// under products: the next tile's scores are formed while this tile's exponentials run.  Against the attention of equal samples, which works on one tile at
// a time, in TFLOP/s: 8192 tokens, 32 heads of 128, no mask 1090 -> 1157, causal 1043 -> 1117; 32 heads of 64, causal 891 -> 938 (a large matrix
// product of this library reaches 1354).
__device__ __forceinline__ float halves_max(float v) {      // of lanes l and l ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
  const unsigned low = r[0], high = r[1];                // (values of their own: a bit cast of a vector's element takes the vector's first)
  return fmaxf(__builtin_bit_cast(float, low), __builtin_bit_cast(float, high));
}
// The weights of a row are exp2(s c2 - m), m its largest s c2 so far, rounded: in one instruction, whose own product is not rounded, so that all of a row's weights
// carry a factor of 2 to the power of m's rounding; their sum and lse carry it too.  From kFar on, where the factor would come to leave 32 bits, rounded products
// that differ at all differ by 32 or more: only those equal to the largest count.  There the scores become the exponents, 0 or -infinity, as soon as
// their maximum mx is known, and m is left out of them.
constexpr float kFar = 0x1p29f;
__device__ __forceinline__ void far_scores(f32x16 (&s)[2], float m_run, float mx, float c2) {
#pragma clang fp contract(off)
  const float m = fmaxf(m_run, mx);
  if (__any(fabsf(m) >= kFar)) {
    const bool far = fabsf(m) >= kFar && m != -INFINITY;
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      const float z = s[e >> 4][e & 15] * c2;
      s[e >> 4][e & 15] = !far ? s[e >> 4][e & 15] : z < m ? -INFINITY : z - m;
      asm volatile("" : "+v"(s[e >> 4][e & 15]));          // (one after the other: side by side they spill)
    }
  }
}
// S^T of the 64 keys of the first stage and a wavefront's 32 queries
template <int D>
__device__ __forceinline__ void fwd_scores(const FragAddr<D>& at, const bf16x8 (&qf)[D / 16], f32x16 (&s)[2]) {
  constexpr int NP = D / 16, kAhead = 3;
  bf16x8 f[kAhead];
  f32x16 zero;
#pragma unroll
  for (int e = 0; e < 16; ++e) zero[e] = 0.f;
#pragma unroll
  for (int i = 0; i < kAhead; ++i) f[i] = at.rows(0, i / NP * 32, i % NP);
  __builtin_amdgcn_sched_barrier(0);
  static_steps<2 * NP>([&](auto step) {
    constexpr int i = decltype(step)::value, b = i / NP, j = i % NP;
    s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], qf[j], j == 0 ? zero : s[b], 0, 0, 0);
    if constexpr (i + kAhead < 2 * NP) f[i % kAhead] = at.rows(0, (i + kAhead) / NP * 32, (i + kAhead) % NP);
    __builtin_amdgcn_sched_barrier(0);
  });
}
__device__ __forceinline__ void hide_scores(f32x16 (&s)[2], int last) {      // key t0 + 32 b + 8 (e / 4) + e % 4 + 4 h is seen up to `last` of that
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) s[b][e] = b * 32 + 8 * (e >> 2) + (e & 3) <= last ? s[b][e] : -INFINITY;
}
// One tile of the forward, its values in stage BUF: its scores are at hand (s, their maximum mx in the log2 domain), and while its exponentials run on the
// vector unit the matrix core forms the next tile's scores (NEXT: keys in the other stage, into nx; mx becomes their maximum) and then
// O^T += V^T P^T.  next_hidden, next_last(): whether some keys of the next tile are hidden, and hide_scores' argument.
// between(i): run after product i; kAhead: products that a fragment is asked for ahead.
template <int D, bool NEXT, int BUF, int kAhead, typename Last, typename Between>
__device__ __forceinline__ void fwd_step(const FragAddr<D>& at, const bf16x8 (&qf)[D / 16], f32x16 (&o)[D / 32], f32x16 (&s)[2], f32x16 (&nx)[2], float& mx, float& m_run,
                                         float& l_run, float c2, bool next_hidden, Last next_last, Between between) {
  constexpr int NP = D / 16, DT = D / 32, NA = NEXT ? 2 * NP : 0, N = NA + 2 * NP;
  auto fetch = [&](int i) -> bf16x8 {
    if (i < NA) return at.rows(2 * (BUF ^ 1), i / NP * 32, i % NP);
    const int k = i - NA, j = k % NP;
    return at.cols(2 * BUF + 1, j % DT, k / NP * 32 + 16 * (j / DT));
  };
  bf16x8 f[kAhead], pf[2][2];
  f32x16 zero;
#pragma unroll
  for (int e = 0; e < 16; ++e) zero[e] = 0.f;
#pragma unroll
  for (int i = 0; i < kAhead; ++i) f[i] = fetch(i);
  __builtin_amdgcn_sched_barrier(0);
  // Running maximum, in the log2 domain.  It is only raised when some row of the wavefront would otherwise see an exponent above 8 (probabilities up to
  // 2^8 are harmless in fp32 / bf16 and cancel in the final division); raising it costs a pass over the output accumulators, and after the
  // first tiles it is rarely needed.
  if (__any(mx > m_run + 8.0f)) {
    const float m_new = fmaxf(m_run, mx);
    const float alpha = (m_new == -INFINITY) ? 1.0f : __builtin_amdgcn_exp2f(m_run - m_new);
    l_run *= alpha;
    m_run = m_new;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[dt][e] *= alpha;
  }
  const float neg_m = fabsf(m_run) < kFar ? -m_run : 0.f;      // (0 for a row without a maximum, too)
  float psum = 0.f, m_next = -INFINITY;
  auto prob = [&](int e) {
    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 4][e & 15], c2, neg_m));
    s[e >> 4][e & 15] = p;
    psum += p;
    asm volatile("" : "+v"(s[e >> 4][e & 15]), "+v"(psum));      // (here, under a product: the compiler would move it behind the branch below)
  };
  if constexpr (!NEXT) {
#pragma unroll
    for (int e = 0; e < 16; ++e) prob(e);
    pf[0][0] = pack8(s[0], 0); pf[0][1] = pack8(s[0], 8);
  }
  static_steps<N>([&](auto step) {
    constexpr int i = decltype(step)::value, k = i - NA;
    if constexpr (i < NA) nx[i / NP] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], qf[i % NP], i % NP == 0 ? zero : nx[i / NP], 0, 0, 0);
    else o[k % NP % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], pf[k / NP][k % NP / DT], o[k % NP % DT], 0, 0, 0);
    if constexpr (i + kAhead < N) f[i % kAhead] = fetch(i + kAhead);
    between(step);
    // the exponentials over the products of the next scores and of the first 32 keys
    if constexpr (NEXT) {
#pragma unroll
      for (int e = i * 32 / (3 * NP); e < (i + 1) * 32 / (3 * NP) && e < 32; ++e) prob(e);
      if constexpr (i == NA - 1) { pf[0][0] = pack8(s[0], 0); pf[0][1] = pack8(s[0], 8); }
    } else if constexpr (i < NP) {
#pragma unroll
      for (int e = 16 + i * 16 / NP; e < 16 + (i + 1) * 16 / NP; ++e) prob(e);
    }
    if constexpr (k == NP - 1) {
      pf[1][0] = pack8(s[1], 0); pf[1][1] = pack8(s[1], 8);
      if (NEXT && next_hidden) hide_scores(nx, next_last());
    }
    if constexpr (NEXT && k >= NP) {
#pragma unroll
      for (int e = (k - NP) * 32 / NP; e < (k - NP + 1) * 32 / NP; ++e) m_next = fmaxf(m_next, nx[e >> 4][e & 15]);
    }
    __builtin_amdgcn_sched_barrier(0);
  });
  l_run += psum;
  if (NEXT) {
    mx = halves_max(m_next) * c2;                        // scores enter the exponent as s * c2 (c2 > 0)
    far_scores(nx, m_run, mx, c2);
  }
}

// A block has 32 QW queries, 32 a wavefront, and KG groups of wavefronts that take every KG-th tile of the keys, in two stages of their own; the groups'
// results are merged at the end.  (4, 1) reads the least from memory and LDS; a launch that leaves compute units idle takes fewer queries a
// block and several groups.
template <int QW, int KG> struct Split {
  static constexpr int THREADS = 64 * QW * KG, ROWS = 32 * QW, PARTS = kPackedTile / ROWS;      // blocks to an entry of the list
  int wave, group, tiles;                              // place in the group, which group, key tiles of the whole block
  __device__ __forceinline__ explicit Split(int ntiles) : tiles(ntiles) {
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    wave = w % QW; group = w / QW;
  }
  __device__ __forceinline__ int at(int i) const { return KG * i + group; }                    // the group's i-th tile
  __device__ __forceinline__ int rounds() const { return (tiles + KG - 1) / KG; }               // of the group with the most
  __device__ __forceinline__ int upto(int n) const { return max(0, (n - group + KG - 1) / KG); } // how many of the group's tiles are below n
};
// the block's entry of the list, head and first query; false: nothing to do
template <int QW, int KG>
__device__ __forceinline__ bool packed_queries(const PackedArgs& p, const PackedOrder& order, int block, PackedTile* e, int* head, int* row0) {
  constexpr int PARTS = Split<QW, KG>::PARTS;
  if constexpr (PARTS == 1) {
    if (!packed_tile(p, order, block, e, head)) return false;
    *row0 = e->tile * kPackedTile;
    return true;
  }
  const int per = order.by_xcd ? 8 * ((order.units + 7) >> 3) : order.units;      // blocks of an entry in the order without parts
  const int rest = block % (PARTS * per), part = uniform(rest / per);
  if (!packed_tile(p, order, block / (PARTS * per) * per + rest % per, e, head)) return false;
  *row0 = e->tile * kPackedTile + (PARTS - 1 - part) * Split<QW, KG>::ROWS;      // (under a mask the last rows have the most keys)
  return *row0 < e->rows;
}

// The loads of the tiles ahead, dealt out over a tile's products: load q of TOTAL follows product q * EVERY.  A load instruction keeps the address unit for 16
// clocks, which the compute unit's wavefronts share: issued in one bunch the eight of a tile of 128 hold a wavefront for 330 to 460 clocks (1024 tokens, 8
// heads of 128 17.1 -> 15.5 us; launches that fill the chip: no difference).
template <int TOTAL, int PRODUCTS, typename Load>
struct Dealt {
  static constexpr int EVERY = PRODUCTS / TOTAL;
  static_assert(EVERY >= 1, "a product for each load");
  Load load;
  template <typename I> __device__ __forceinline__ void operator()(I) const {
    if constexpr (I::value % EVERY == 0 && I::value / EVERY < TOTAL) load(I::value / EVERY);
  }
};
template <int TOTAL, int PRODUCTS, typename Load> __device__ __forceinline__ Dealt<TOTAL, PRODUCTS, Load> dealt(Load load) { return {load}; }
// the descriptor, or one of no extent: its loads bring zeros
__device__ __forceinline__ i32x4 only_if(bool there, i32x4 rsrc) { return i32x4{rsrc[0], rsrc[1], there ? rsrc[2] : 0, rsrc[3]}; }

// The keys are staged one tile further ahead than the values.  The queries of a wavefront see the group's first `mine` tiles; it helps to stage the others.
template <int D, bool CAUSAL, int QW, int KG>
__global__ void __launch_bounds__(64 * QW * KG, (KG == 1 ? kFwdWaves<D> : D == 128 ? 1 : 2))
packed_fwd_kernel(PackedArgs p, PackedOrder order, const bf16* __restrict__ qkv, bf16* __restrict__ O, float* __restrict__ lse) {
  const int block = blockIdx.x;
  typedef Tile<D, TILE, 64 * QW> TL;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  PackedTile e;
  int a, r0;
  if (!packed_queries<QW, KG>(p, order, block, &e, &a, &r0)) return;
  const int lane = threadIdx.x & 63;
  const int S = e.rows, d = p.d, g = a / p.group;
  const SampleRows x(qkv, p.ld, e.first, S, (p.heads + 2 * p.kv_heads) * d);
  const unsigned k_bytes = (unsigned)((p.heads + g) * d * 2), v_bytes = k_bytes + (unsigned)(p.kv_heads * d * 2);
  const float c2 = p.scale * kLog2e;
  const Split<QW, KG> grp(((CAUSAL ? min(S, r0 + 32 * QW) : S) + TILE - 1) / TILE);
  const int q0 = r0 + grp.wave * 32;
  lds_bf16* smem = (lds_bf16*)smem_raw + grp.group * 4 * TL::ELEMS;
  auto Ks = [&](int st) { return smem + st * 2 * TL::ELEMS; };
  auto Vs = [&](int st) { return smem + st * 2 * TL::ELEMS + TL::ELEMS; };

  bf16x8 qf[D / 16];
  load_row_frags<D>(x.base + a * d, p.ld, q0, S, qf, d);
  unsigned part[TL::PER_WAVE];
  TL::stage_lanes(part, x.ld_bytes, d, grp.wave);
  const unsigned tile_bytes = TILE * x.ld_bytes;
  auto stage_keys = [&](int i) { if (grp.at(i) < grp.tiles) TL::stage_at(x.rsrc, part, (unsigned)grp.at(i) * tile_bytes + k_bytes, Ks(i & 1), grp.wave); };
  auto stage_values = [&](int i) { if (grp.at(i) < grp.tiles) TL::stage_at(x.rsrc, part, (unsigned)grp.at(i) * tile_bytes + v_bytes, Vs(i & 1), grp.wave); };
  auto close = [&] {
    __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0): this wavefront's rows have landed
    __syncthreads();
  };
  stage_keys(0);
  stage_keys(1);
  stage_values(0);
  close();

  FragAddr<D> at(smem);
  at.hold();
  f32x16 o[D / 32], s0[2], s1[2];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f, mx = -INFINITY;
  const int rounds = grp.rounds(), mine = q0 >= S ? 0 : grp.upto(CAUSAL ? min(grp.tiles, (q0 + 31) / TILE + 1) : grp.tiles);
  // the last key that the lane's query sees, counted from the lane's first of tile kt on (formed where it is used: kept, it is a register too many)
  auto last = [&](int kt) {
    int l = threadIdx.x & 63;
    asm volatile("" : "+v"(l));
    return (CAUSAL ? min(q0 + (l & 31), S - 1) : S - 1) - 4 * (l >> 5) - kt * TILE;
  };
  auto hidden = [&](int kt) { return (CAUSAL && kt * TILE + 63 > q0) || kt * TILE + 64 > S; };
  if (mine > 0) {
    fwd_scores<D>(at, qf, s0);
    if (hidden(grp.at(0))) hide_scores(s0, last(grp.at(0)));
#pragma unroll
    for (int i = 0; i < 32; ++i) mx = fmaxf(mx, s0[i >> 4][i & 15]);
    mx = halves_max(mx) * c2;
    far_scores(s0, m_run, mx, c2);
  }
  __syncthreads();                                       // (every wavefront has its scores of tile 0: the keys of tile 2 take its place)
  int i = 0;
  auto step = [&](auto next, auto buf, auto ahead, f32x16 (&s)[2], f32x16 (&nx)[2]) {
    const int kt = grp.at(i + 1), kt2 = grp.at(i + 2);
    const i32x4 keys = only_if(kt2 < grp.tiles, x.rsrc), values = only_if(kt < grp.tiles, x.rsrc);
    auto loads = dealt<2 * TL::PER_WAVE, (decltype(next)::value ? 4 : 2) * D / 16>([&](int n) {
      constexpr int B = decltype(buf)::value;
      if (n < TL::PER_WAVE) TL::stage_one_at(keys, part[n], (unsigned)kt2 * tile_bytes + k_bytes, Ks(B), grp.wave, n);
      else TL::stage_one_at(values, part[n - TL::PER_WAVE], (unsigned)kt * tile_bytes + v_bytes, Vs(B ^ 1), grp.wave, n - TL::PER_WAVE);
    });
    fwd_step<D, decltype(next)::value, decltype(buf)::value, decltype(ahead)::value>(at, qf, o, s, nx, mx, m_run, l_run, c2, hidden(kt), [&] { return last(kt); }, loads);
    close();
    ++i;
  };
  const std::true_type more;
  const std::false_type end;
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  const std::integral_constant<int, 3> three;
  const std::integral_constant<int, 2> two;              // (three spill a register behind the loop)
  while (i + 2 < mine) {
    step(more, even, three, s0, s1);
    step(more, odd, three, s1, s0);
  }
  if (i + 1 < mine) {
    step(more, even, two, s0, s1);
    step(end, odd, two, s1, s0);
  } else if (i < mine) {
    step(end, even, two, s0, s1);
  }
  for (; i < rounds; ++i) {
    stage_keys(i + 2);
    stage_values(i + 1);
    close();
  }
  if constexpr (KG > 1) {                                // [value][lane] floats of each wavefront behind the first group's, lanes next to one another
    constexpr int NV = D / 32 * 16 + 2;
    LDS_AS float* mrg = (LDS_AS float*)smem_raw + lane;
    if (grp.group > 0) {
      LDS_AS float* to = mrg + ((grp.group - 1) * QW + grp.wave) * NV * 64;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) to[(dt * 16 + i) * 64] = o[dt][i];
      to[(NV - 2) * 64] = m_run;
      to[(NV - 1) * 64] = l_run;
    }
    __syncthreads();
    if (grp.group > 0) return;
#pragma unroll
    for (int other = 0; other < KG - 1; ++other) {
      const LDS_AS float* from = mrg + (other * QW + grp.wave) * NV * 64;
      const float m1 = from[(NV - 2) * 64], m = fmaxf(m_run, m1);
      const float a0 = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m), a1 = m1 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m1 - m);
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = o[dt][i] * a0 + from[(dt * 16 + i) * 64] * a1;
      l_run = l_run * a0 + from[(NV - 1) * 64] * a1;
      m_run = m;
    }
  }
  const float l_tot = l_run + __shfl_xor(l_run, 32, 64);
  int at_lane = threadIdx.x & 63;
  asm volatile("" : "+v"(at_lane));                      // (formed again here, not kept through the loop)
  const int q = q0 + (at_lane & 31);
  store_transposed<D>(o, O + (int64_t)e.first * p.ldo + a * d, p.ldo, q, S, 1.0f / l_tot, d);
  if (at_lane < 32 && q < S) lse[(int64_t)a * p.tokens + e.first + q] = (m_run + __builtin_amdgcn_logf(l_tot)) * kLn2;
}

// ------------------------------------------------------------------------------------ dQ
// dvec: where rowsum(dO O) goes for the dK / dV blocks, or null
template <int D, bool CAUSAL, int QW, int KG>
__device__ __forceinline__ void dq_block(const PackedArgs& p, const PackedOrder& order, int block, const bf16* __restrict__ qkv, const bf16* __restrict__ O,
                                         const bf16* __restrict__ dO, const float* __restrict__ lse, float* __restrict__ dvec, bf16* __restrict__ dqkv) {
  typedef Tile<D, TILE, 64 * QW> TL;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  PackedTile e;
  int a, r0;
  if (!packed_queries<QW, KG>(p, order, block, &e, &a, &r0)) return;
  const int lane = threadIdx.x & 63, h = lane >> 5;
  const int S = e.rows, d = p.d, g = a / p.group;
  const SampleRows x(qkv, p.ld, e.first, S, (p.heads + 2 * p.kv_heads) * d);
  const unsigned k_bytes = (unsigned)((p.heads + g) * d * 2), v_bytes = k_bytes + (unsigned)(p.kv_heads * d * 2);
  const float c2 = p.scale * kLog2e;
  const Split<QW, KG> grp(((CAUSAL ? min(S, r0 + 32 * QW) : S) + TILE - 1) / TILE);
  const int q0 = r0 + grp.wave * 32, q = q0 + (lane & 31);
  lds_bf16* smem = (lds_bf16*)smem_raw + grp.group * 4 * TL::ELEMS;
  auto Ks = [&](int st) { return smem + st * 2 * TL::ELEMS; };
  auto Vs = [&](int st) { return smem + st * 2 * TL::ELEMS + TL::ELEMS; };

  unsigned part[TL::PER_WAVE];
  TL::stage_lanes(part, x.ld_bytes, d, grp.wave);
  const unsigned tile_bytes = TILE * x.ld_bytes;
  auto stage = [&](int i) {
    if (grp.at(i) >= grp.tiles) return;
    const unsigned rows = (unsigned)grp.at(i) * tile_bytes;
    TL::stage_at(x.rsrc, part, rows + k_bytes, Ks(i & 1), grp.wave);
    TL::stage_at(x.rsrc, part, rows + v_bytes, Vs(i & 1), grp.wave);
  };
  auto close = [&] {
    __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0)
    __syncthreads();
  };
  stage(0);
  bf16x8 qf[D / 16], dof[D / 16];
  const int64_t orow = (int64_t)e.first * p.ldo + a * d, stat = (int64_t)a * p.tokens + e.first + q;
  load_row_frags<D>(dO + orow, p.ldo, q0, S, dof, d);
  const float dv = row_dot<D>(O + orow, p.ldo, q0, S, dof, d);
  load_row_frags<D>(x.base + a * d, p.ld, q0, S, qf, d);
  const float lse2 = q < S ? lse[stat] * kLog2e : 0.f;
  if (dvec && h == 0 && q < S && grp.group == 0) dvec[stat] = dv;
  f32x16 dq[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) dq[dt][i] = 0.f;
  close();
  FragAddr<D> at(smem);
  const int rounds = grp.rounds(), mine = q0 >= S ? 0 : grp.upto(CAUSAL ? min(grp.tiles, (q0 + 31) / TILE + 1) : grp.tiles);
  const int limit = (CAUSAL ? min(q, S - 1) : S - 1) - 4 * h;      // the last key that the lane's query sees
  int i = 0;
  for (; i < mine; ++i) {
    const int t0 = grp.at(i) * TILE, kt = grp.at(i + 1), st = (i + 1) & 1;
    const i32x4 ahead = only_if(kt < grp.tiles, x.rsrc);
    auto loads = dealt<2 * TL::PER_WAVE, 6 * D / 16>([&](int n) {
      const int j = n % TL::PER_WAVE;
      TL::stage_one_at(ahead, part[j], (unsigned)kt * tile_bytes + (n < TL::PER_WAVE ? k_bytes : v_bytes), n < TL::PER_WAVE ? Ks(st) : Vs(st), grp.wave, j);
    });
    dq_tile<D, 0>(at, qf, dof, dq, c2, lse2, dv, (CAUSAL && t0 + 63 > q0) || t0 + 64 > S, limit - t0, loads);
    at.flip();
    close();
  }
  for (; i < rounds; ++i) {
    stage(i + 1);
    close();
  }
  if constexpr (KG > 1) {
    LDS_AS float* mrg = (LDS_AS float*)smem_raw + lane;
    if (grp.group > 0) {
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) mrg[(((grp.group - 1) * QW + grp.wave) * (D / 32 * 16) + dt * 16 + i) * 64] = dq[dt][i];
    }
    __syncthreads();
    if (grp.group > 0) return;
#pragma unroll
    for (int other = 0; other < KG - 1; ++other)
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[dt][i] += mrg[((other * QW + grp.wave) * (D / 32 * 16) + dt * 16 + i) * 64];
  }
  store_transposed<D>(dq, dqkv + (int64_t)e.first * p.ld + a * d, p.ld, q, S, p.scale, d);
}

template <int D, bool CAUSAL>
__global__ void __launch_bounds__(kThreads, kDqWaves<D>)
packed_dq_kernel(PackedArgs p, PackedOrder order, const bf16* __restrict__ qkv, const bf16* __restrict__ O, const bf16* __restrict__ dO,
                 const float* __restrict__ lse, float* __restrict__ dvec, bf16* __restrict__ dqkv) {
  dq_block<D, CAUSAL, 4, 1>(p, order, blockIdx.x, qkv, O, dO, lse, dvec, dqkv);
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

// rowsum(dO O) of a tile of 64 rows: asked for with the tile, formed when it has landed.  THREADS / 64 threads to a row.
template <int D, int THREADS> struct OwnRows {
  static constexpr int PER = THREADS / TILE, N = D / PER / 8;                // 16-byte pieces of a thread
  bf16x8 o[N], g[N];
  __device__ __forceinline__ void load(const bf16* __restrict__ O, const bf16* __restrict__ dO, const PackedArgs& p, const KeyItem& e, int head, int row0) {
    const int r = row0 + threadIdx.x / PER, c0 = threadIdx.x % PER * (D / PER);
    const int64_t at = ((int64_t)e.first + r) * p.ldo + head * p.d + c0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      o[k] = g[k] = bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
      if (r < e.rows && c0 + 8 * k < p.d) {
        o[k] = *reinterpret_cast<const bf16x8*>(O + at + 8 * k);
        g[k] = *reinterpret_cast<const bf16x8*>(dO + at + 8 * k);
      }
    }
  }
  __device__ __forceinline__ void store(LDS_AS float* to, float sign) const {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) v = __builtin_fmaf((float)o[k][i], (float)g[k][i], v);
#pragma unroll
    for (int s = 1; s < PER; s *= 2) v += __shfl_xor(v, s, 64);
    if (threadIdx.x % PER == 0) to[threadIdx.x / PER] = sign * v;
  }
};

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
  if (!rows_fit(p, e.first, e.rows, e.tile) || t >= e.rows || d0 >= p.d || e.slot < 0 || e.pieces > p.slots - e.slot) return;
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
// OWN: rowsum(dO O) is formed here, from O, not read from dvec.
template <int D, bool CAUSAL, bool OWN>
__device__ __forceinline__ void dkv_narrow_block(const PackedArgs& p, const PackedOrder& order, int block, const bf16* __restrict__ qkv, const bf16* __restrict__ O,
                                                 const bf16* __restrict__ dO, const float* __restrict__ lse, const float* __restrict__ dvec, bf16* __restrict__ dqkv) {
  typedef Tile<D> TL;
  extern __shared__ __attribute__((aligned(16))) char smem_raw[];
  lds_bf16* smem = (lds_bf16*)smem_raw;
  auto Qs = [&](int st) { return smem + st * 2 * TL::ELEMS; };
  auto dOs = [&](int st) { return smem + st * 2 * TL::ELEMS + TL::ELEMS; };
  LDS_AS float* stats = (LDS_AS float*)(smem + 4 * TL::ELEMS);      // [2 buffers][-lse / scale | -dvec][64]
  KeyItem e;
  int g;
  if (!packed_keys(p, order, block, CAUSAL, &e, &g)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, h = lane >> 5;
  const int S = e.rows, d = p.d, a0 = g * p.group;
  const SampleRows x(qkv, p.ld, e.first, S, (p.heads + 2 * p.kv_heads) * d), y(dO, p.ldo, e.first, S, p.heads * d);
  const float c2 = p.scale * kLog2e, per_scale = -1.0f / p.scale;
  const int t0 = e.tile * 128 + wave * 32, t = t0 + (lane & 31);

  QueryWalk next(e, CAUSAL, p.group), now = next;
  int buf = 0;                                         // where the next tile goes
  float rstat = 0.f;                                   // threads 0..63: of lse, 64..127: of dvec
  OwnRows<D, kThreads> own;
  constexpr float kSign = -1.0f;
  auto stage_next = [&] {
    if (!next.more()) return;
    const unsigned col = (unsigned)((a0 + next.head) * d * 2);
    TL::stage(x.rsrc, col, x.ld_bytes, next.it * TILE, Qs(buf), d);
    TL::stage(y.rsrc, col, y.ld_bytes, next.it * TILE, dOs(buf), d);
    rstat = 0.f;
    const int r = next.it * TILE + (threadIdx.x & 63);
    if (threadIdx.x < (OWN ? 64 : 128) && r < S) {
      const int64_t at = (int64_t)(a0 + next.head) * p.tokens + e.first + r;
      rstat = threadIdx.x < 64 ? lse[at] * per_scale : -dvec[at];
    }
    if constexpr (OWN) own.load(O, dO, p, e, a0 + next.head, next.it * TILE);
  };
  auto close = [&] {                                   // the tile that was staged becomes the current one
    if (next.more()) {
      if (threadIdx.x < (OWN ? 64 : 128)) stats[buf * 128 + threadIdx.x] = rstat;
      if constexpr (OWN) own.store(stats + buf * 128 + 64, kSign);
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
template <int D, bool CAUSAL, bool OWN>
__device__ __forceinline__ void dkv_wide_block(const PackedArgs& p, const PackedOrder& order, int block, const bf16* __restrict__ qkv, const bf16* __restrict__ O,
                                               const bf16* __restrict__ dO, const float* __restrict__ lse, const float* __restrict__ dvec, bf16* __restrict__ dqkv) {
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
  if (!packed_keys(p, order, block, CAUSAL, &e, &g)) return;
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
  OwnRows<D, kThreads8> own;
  constexpr float kSign = 1.0f;
  auto stage_next = [&] {
    if (!next.more()) return;
    const unsigned col = (unsigned)((a0 + next.head) * d * 2);
    TL::stage(x.rsrc, col, x.ld_bytes, next.it * TILE, Qs(buf), d);
    TL::stage(y.rsrc, col, y.ld_bytes, next.it * TILE, dOs(buf), d);
    rstat = 0.f;
    const int r = next.it * TILE + (threadIdx.x & 63);
    if (threadIdx.x < (OWN ? 64 : 128) && r < S) {
      const int64_t at = (int64_t)(a0 + next.head) * p.tokens + e.first + r;
      rstat = threadIdx.x < 64 ? lse[at] * kLog2e : dvec[at];
    }
    if constexpr (OWN) own.load(O, dO, p, e, a0 + next.head, next.it * TILE);
  };
  auto close = [&] {
    if (next.more()) {
      if (threadIdx.x < (OWN ? 64 : 128)) stats[buf * 128 + threadIdx.x] = rstat;
      if constexpr (OWN) own.store(stats + buf * 128 + 64, kSign);
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
__global__ void __launch_bounds__(kThreads, kDkvWaves<D>)
packed_dkv_narrow_kernel(PackedArgs p, PackedOrder order, const bf16* __restrict__ qkv, const bf16* __restrict__ dO, const float* __restrict__ lse,
                         const float* __restrict__ dvec, bf16* __restrict__ dqkv) {
  dkv_narrow_block<D, CAUSAL, false>(p, order, blockIdx.x, qkv, nullptr, dO, lse, dvec, dqkv);
}
template <int D, bool CAUSAL>
__global__ void __launch_bounds__(kThreads8, 2)
packed_dkv_kernel(PackedArgs p, PackedOrder order, const bf16* __restrict__ qkv, const bf16* __restrict__ dO, const float* __restrict__ lse,
                  const float* __restrict__ dvec, bf16* __restrict__ dqkv) {
  dkv_wide_block<D, CAUSAL, false>(p, order, blockIdx.x, qkv, nullptr, dO, lse, dvec, dqkv);
}
// The whole backward in one launch, where one after the other its two halves would leave compute units idle: the blocks of dK and dV, the longer ones, first.
// They form rowsum(dO O) themselves.
template <int D> constexpr int kBothThreads = D <= 64 ? kThreads : kThreads8;
template <int D, bool CAUSAL>
__global__ void __launch_bounds__(kBothThreads<D>, 2)
packed_bwd_kernel(PackedArgs p, PackedOrder by_keys, PackedOrder by_queries, int key_blocks, const bf16* __restrict__ qkv, const bf16* __restrict__ O,
                  const bf16* __restrict__ dO, const float* __restrict__ lse, bf16* __restrict__ dqkv) {
  const int block = blockIdx.x;
  if (block >= key_blocks) dq_block<D, CAUSAL, D <= 64 ? 2 : 4, 2>(p, by_queries, block - key_blocks, qkv, O, dO, lse, nullptr, dqkv);
  else if constexpr (D <= 64) dkv_narrow_block<D, CAUSAL, true>(p, by_keys, block, qkv, O, dO, lse, nullptr, dqkv);
  else dkv_wide_block<D, CAUSAL, true>(p, by_keys, block, qkv, O, dO, lse, nullptr, dqkv);
}

template <int D, bool CAUSAL, int QW, int KG>
int launch_fwd(const PackedArgs& a, const bf16* qkv, bf16* O, float* lse, hipStream_t s) {
  PackedOrder order;
  const unsigned grid = packed_grid(a.tiles, a.heads, &order) * Split<QW, KG>::PARTS;
  constexpr auto kern = packed_fwd_kernel<D, CAUSAL, QW, KG>;
  constexpr size_t lds = KG * 4 * (size_t)Tile<D>::ELEMS * sizeof(bf16), merge = (size_t)(KG - 1) * QW * (D / 32 * 16 + 2) * 64 * sizeof(float);
  static_assert(merge <= lds && lds <= 160 * 1024, "the merge takes the stages' place");
  if (const int rc = reserve_lds<kern>("attention_packed", lds); rc != CEPHALO_OK) return rc;
  kern<<<grid, Split<QW, KG>::THREADS, lds, s>>>(a, order, qkv, O, lse);
  CEPHALO_CHECK_LAUNCH("attention_packed_fwd");
  return CEPHALO_OK;
}
template <int D, bool CAUSAL>
int launch_dq(const PackedArgs& a, const bf16* qkv, const bf16* O, const bf16* dO, const float* lse, float* dvec, bf16* dqkv, hipStream_t s) {
  PackedOrder order;
  const unsigned grid = packed_grid(a.tiles, a.heads, &order);
  constexpr auto kern = packed_dq_kernel<D, CAUSAL>;
  constexpr size_t lds = 4 * (size_t)Tile<D>::ELEMS * sizeof(bf16);
  if (const int rc = reserve_lds<kern>("attention_packed", lds); rc != CEPHALO_OK) return rc;
  kern<<<grid, kThreads, lds, s>>>(a, order, qkv, O, dO, lse, dvec, dqkv);
  CEPHALO_CHECK_LAUNCH("attention_packed_dq");
  return CEPHALO_OK;
}
// Whether a forward takes the form (2, 2): where 128 queries a block would leave half of the compute units without one (heads up to 64, two of whose blocks
// share a compute unit: some of them).  Us of the forward, (4, 1) and (2, 2), by list entries times heads.  Heads of 128: 64: 21 and 16; 128: 21 and 17;
// 256: 24 and 25 (2 x 1024 tokens), 36 and 34 (2048, 16 key heads); 384: 42 and 50; 512 (8 x 512, no mask): 26 and 45.  Heads of 64: 32: 10.4 and 8.3;
// 256: 26 and 20 (2048 tokens), 10.6 and 9.0 (8 x 512); 384: 13.8 and 16.1; 512: 10.9 and 14.5.
bool halves(const PackedArgs& a, int D) { return (int64_t)a.tiles * a.heads <= (D <= 64 ? 256 : 128); }

template <int D, bool CAUSAL>
int fwd_cfg(const PackedArgs& a, const bf16* qkv, bf16* O, float* lse, hipStream_t s) {
  return halves(a, D) ? launch_fwd<D, CAUSAL, 2, 2>(a, qkv, O, lse, s) : launch_fwd<D, CAUSAL, 4, 1>(a, qkv, O, lse, s);
}

template <int D> int join(const PackedArgs& a, bf16* dqkv, hipStream_t s) {
  if (a.join_items == 0) return CEPHALO_OK;
  packed_join_kernel<D><<<dim3(D / 4, a.join_items, a.kv_heads), 256, 0, s>>>(a, dqkv);
  CEPHALO_CHECK_LAUNCH("attention_packed_join");
  return CEPHALO_OK;
}

template <int D, bool CAUSAL>
int bwd_cfg(const PackedArgs& a, const bf16* qkv, const bf16* O, const bf16* dO, const float* lse, float* dvec, bf16* dqkv, hipStream_t s) {
  // two stages of Q and dO (and, wide, the keys and values) and of the row statistics, or at the end the merge of the halves
  constexpr size_t stages = (4 * (size_t)Tile<D>::ELEMS + (D <= 64 ? 0 : 2 * (size_t)Tile<D, 128>::ELEMS)) * sizeof(bf16) + 2 * 128 * sizeof(float);
  constexpr size_t merge = D <= 64 ? 0 : (size_t)4 * (D / 32 * 16 * 2) * 64 * sizeof(float);
  constexpr size_t lds = stages > merge ? stages : merge;
  PackedOrder order;
  const unsigned key_blocks = packed_grid(a.key_items, a.kv_heads, &order);
  if (packed_one_launch(a.tiles, a.heads, a.kv_heads, a.d)) {
    PackedOrder by_queries;
    constexpr int PARTS = Split<D <= 64 ? 2 : 4, 2>::PARTS;
    const unsigned query_blocks = packed_grid(a.tiles, a.heads, &by_queries) * PARTS;
    constexpr auto kern = packed_bwd_kernel<D, CAUSAL>;
    constexpr size_t dq_lds = 8 * (size_t)Tile<D>::ELEMS * sizeof(bf16), most = dq_lds > lds ? dq_lds : lds;
    if (const int rc = reserve_lds<kern>("attention_packed", most); rc != CEPHALO_OK) return rc;
    kern<<<key_blocks + query_blocks, kBothThreads<D>, most, s>>>(a, order, by_queries, (int)key_blocks, qkv, O, dO, lse, dqkv);
    CEPHALO_CHECK_LAUNCH("attention_packed_bwd");
    return join<D>(a, dqkv, s);
  }
  if (const int rc = launch_dq<D, CAUSAL>(a, qkv, O, dO, lse, dvec, dqkv, s); rc != CEPHALO_OK) return rc;
  if constexpr (D <= 64) {
    constexpr auto kern = packed_dkv_narrow_kernel<D, CAUSAL>;
    if (const int rc = reserve_lds<kern>("attention_packed", lds); rc != CEPHALO_OK) return rc;
    kern<<<key_blocks, kThreads, lds, s>>>(a, order, qkv, dO, lse, dvec, dqkv);
  } else {
    constexpr auto kern = packed_dkv_kernel<D, CAUSAL>;
    if (const int rc = reserve_lds<kern>("attention_packed", lds); rc != CEPHALO_OK) return rc;
    kern<<<key_blocks, kThreads8, lds, s>>>(a, order, qkv, dO, lse, dvec, dqkv);
  }
  CEPHALO_CHECK_LAUNCH("attention_packed_dkv");
  return join<D>(a, dqkv, s);
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
