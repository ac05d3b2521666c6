// What the bf16 attention kernels share: operand tiles in LDS, fragments, the products of one wavefront's share of a tile, transposed stores.
#pragma once
#include <type_traits>
#include <utility>
#include "kernels.h"

namespace cephalo {
namespace {

typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
#define LDS_AS __attribute__((address_space(3)))
typedef LDS_AS bf16 lds_bf16;

constexpr int kThreads = 256;
constexpr int TILE = 64;            // tokens per LDS tile
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* p, unsigned bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}
// the same descriptor as four words (base, base high half with stride 0, extent, flags), for inline assembly
typedef int i32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ i32x4 make_rsrc_words(const void* p, unsigned bytes) {
  const uint64_t addr = (uint64_t)(uintptr_t)p;
  return i32x4{(int)(unsigned)addr, (int)(unsigned)((addr >> 32) & 0xffffu), (int)bytes, 0x00020000};
}

// ROWS tokens by D values (D = 32, 64 or 128) of one operand in LDS, staged by THREADS threads straight from global memory.
//
// Rows are 2 D bytes without padding, so that a direct-to-LDS load of 16 bytes per lane fills 1 KiB = 512 / D whole rows at once; bank
// conflicts are avoided by permuting the 16-byte chunks of a row, chunk c of row r lives at chunk  c ^ swz(r);  the permutation is
// applied by the address each lane fetches.  16 consecutive rows put the same chunk on 16 different places of the 64 banks (fragment
// reads: 1, 2 or 4 rows share a line of all banks), and 4 consecutive rows put four neighbouring chunks on disjoint places
// (transposing reads):
//     D = 128   swz(r) = ((r & 7) << 1) | ((r >> 3) & 1)
//     D =  64   swz(r) = (((r >> 1) & 1) << 2) | ((r >> 2) & 3)
//     D =  32   swz(r) = (r >> 2) & 3
// (With padded rows only 4-byte-per-lane loads fit a row, and those run at a quarter of the rate; through registers, as the
// 64-wide tiles used to be staged, the loads cost 16 registers and an LDS write each.)
template <int D, int ROWS = TILE, int THREADS = kThreads> struct Tile {
  static constexpr int LD = D;
  static constexpr int ELEMS = ROWS * LD;
  __device__ static constexpr int swz(int r) {
    return D == 128 ? ((r & 7) << 1) | ((r >> 3) & 1) : D == 64 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : (r >> 2) & 3;
  }
  static constexpr int FLIP8 = D == 128 ? 1 : 2;          // swz(r + 8) = swz(r) ^ FLIP8 for r < 8

  // rsrc covers exactly one sample of the [*, ld_bytes/2] matrix, col_bytes is the head's
  // column offset.  Rows past the sample's end and chunks past the head's own width d are beyond the buffer's range
  // (every part of the address is in the range-checked offset): the hardware makes them zeros; callers mask such keys.
  // The loads are asynchronous: wait for vmcnt(0) and a workgroup barrier before reading the tile.
  static constexpr int NW = THREADS / 64, RPL = 512 / D, LOADS = ROWS / RPL, PER_WAVE = LOADS >= NW ? LOADS / NW : 1;      // RPL: rows per load
  static_assert(LOADS % NW == 0 || NW % LOADS == 0, "loads split evenly over the wavefronts");
  // the part of the offset that belongs to the lane (the same for every tile: the compiler keeps it out of the loops)
  // (wave: this wavefront's place among the THREADS / 64 that stage the tile; by default its place in the block)
  __device__ static unsigned stage_lane(int j, unsigned ld_bytes, int d, int wave = -1) {
    if (wave < 0) wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int row = (wave * PER_WAVE + j) * RPL + lane / (D / 8);
    const int c = (lane % (D / 8)) ^ swz(row);
    return c * 8 < d ? (unsigned)row * ld_bytes + (unsigned)c * 16 : 0x80000000u;
  }
  // The loads are issued behind the compiler's back: it tracks loads that write LDS, cannot tell one buffer from
  // another, and makes later LDS reads of the tile being multiplied wait for them (the whole memory latency, every
  // tile).  Callers wait (vmcnt(0)) and synchronise before they read what was staged.
  __device__ static void stage_one(i32x4 rsrc, int j, unsigned tile_bytes, unsigned ld_bytes, lds_bf16* lds, int d) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (LOADS < NW && wave >= LOADS) return;               // (a tile with fewer loads than wavefronts)
    const unsigned dst = (unsigned)(uintptr_t)(lds + (wave * PER_WAVE + j) * RPL * LD);
    const unsigned off = stage_lane(j, ld_bytes, d) + tile_bytes;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(dst), "v"(off), "s"(rsrc) : "m0");
  }
  __device__ static void stage(i32x4 rsrc, unsigned col_bytes, unsigned ld_bytes, int row0, lds_bf16* lds, int d) {
#pragma unroll
    for (int j = 0; j < PER_WAVE; ++j) stage_one(rsrc, j, (unsigned)row0 * ld_bytes + col_bytes, ld_bytes, lds, d);
  }
  // The same with the lanes' parts of the offsets at hand (wave: this wavefront's place among those that stage the tile).
  __device__ static __forceinline__ void stage_lanes(unsigned (&part)[PER_WAVE], unsigned ld_bytes, int d, int wave) {
#pragma unroll
    for (int j = 0; j < PER_WAVE; ++j) {
      part[j] = stage_lane(j, ld_bytes, d, wave);
      asm volatile("" : "+v"(part[j]));                    // (kept: formed again for every tile they cost more than the products leave time for)
    }
  }
  __device__ static __forceinline__ void stage_one_at(i32x4 rsrc, unsigned part, unsigned tile_bytes, lds_bf16* lds, int wave, int j) {
    if (LOADS < NW && wave >= LOADS) return;
    const unsigned dst = (unsigned)(uintptr_t)(lds + (wave * PER_WAVE + j) * RPL * LD), off = part + tile_bytes;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(dst), "v"(off), "s"(rsrc) : "m0");
  }
  __device__ static __forceinline__ void stage_at(i32x4 rsrc, const unsigned (&part)[PER_WAVE], unsigned tile_bytes, lds_bf16* lds, int wave) {
#pragma unroll
    for (int j = 0; j < PER_WAVE; ++j) stage_one_at(rsrc, part[j], tile_bytes, lds, wave, j);
  }
  // operand with MFMA rows = tile rows [rb, rb+32), contraction over d in [kk, kk+16)   (rb: a multiple of 16 rows from
  // the tile's first row, so that a row's place in its group of 16 is the lane's)
  __device__ static bf16x8 frag_rows(const lds_bf16* lds, int rb, int kk) {
    const int lane = threadIdx.x & 63;
    // chunk (kk/8 + h) ^ swz = (kk/8) ^ (h ^ swz): the lane's part once, the fragment's part as an XOR of the byte address
    const unsigned own = (unsigned)(lane & 31) * (LD * 2) + (unsigned)(((lane >> 5) ^ swz(lane & 15)) << 4);
    return *reinterpret_cast<const LDS_AS bf16x8*>((const LDS_AS char*)lds + rb * (LD * 2) + (own ^ (unsigned)(kk * 2)));
  }
  // operand with MFMA rows = d in [db, db+32), contraction over 16 tile rows in the order the
  // accumulator of a preceding 32x32 product holds them: slot 4c+i of half-wave h is tile row
  // tb + 8c + 4h + i  (tb = first of the 16 rows, a multiple of 16 rows from the tile's first row)
  __device__ static bf16x8 frag_cols(const lds_bf16* lds, int db, int tb) {
    const int lane = threadIdx.x & 63;
    const int g = lane >> 4, i = lane & 15;
    // rows r and r + 8 (r < 8): the second read is the first with a chunk bit flipped
    const int r = 4 * (g >> 1) + (i >> 2);
    const unsigned own = (unsigned)r * (LD * 2) + (unsigned)(((2 * (g & 1) + ((i & 3) >> 1)) ^ swz(r)) << 4) + 8u * (i & 1);
    const LDS_AS char* p0 = (const LDS_AS char*)lds + tb * (LD * 2);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(p0 + (own ^ (unsigned)(db * 2))));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(p0 + 8 * (LD * 2) + ((own ^ (16u * FLIP8)) ^ (unsigned)(db * 2))));
    union { struct { s16x4 a, b; } s; bf16x8 v; } u;
    u.s.a = lo; u.s.b = hi;
    return u.v;
  }
};

// The LDS addresses of one lane's fragment reads (Tile::frag_rows / frag_cols) for two double-buffered tiles A and B that lie [A | B][A | B]: a register
// per constant that the permutation XORs in, everything else in the instruction's offset, and one XOR each to turn to the other buffer.
// (Left to itself the compiler keeps an address per constant and buffer, or forms one per read, an instruction beside every product.)
template <int D> struct FragAddr {
  typedef Tile<D> TL;
  static constexpr unsigned TILE_BYTES = TL::ELEMS * 2, STAGE = 2 * TILE_BYTES;
  unsigned r[D / 16], lo[D / 32], hi[D / 32];
  __device__ __forceinline__ explicit FragAddr(const lds_bf16* first) {
    // The XORs need a multiple of 2 * STAGE.  The tiles are the first of the dynamic LDS, which begins at 0 as long as the kernel has no static LDS: a test
    // of the compiled kernels sees to that.
    const unsigned base = (unsigned)(uintptr_t)first;
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                       // (formed here, not kept from pass to pass)
    const int g = lane >> 4, i = lane & 15, row = 4 * (g >> 1) + (i >> 2);
    const unsigned rows = (unsigned)(lane & 31) * (D * 2) + (unsigned)(((lane >> 5) ^ TL::swz(lane & 15)) << 4);
    const unsigned cols = (unsigned)row * (D * 2) + (unsigned)(((2 * (g & 1) + ((i & 3) >> 1)) ^ TL::swz(row)) << 4) + 8u * (i & 1);
#pragma unroll
    for (int k = 0; k < D / 16; ++k) r[k] = base + (rows ^ (unsigned)(k * 32));
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      lo[k] = base + (cols ^ (unsigned)(k * 64));
      hi[k] = base + (cols ^ (16u * TL::FLIP8) ^ (unsigned)(k * 64));
    }
  }
  __device__ __forceinline__ void hold() {               // (the addresses as they are: the compiler would add `first` again at every read)
#pragma unroll
    for (int k = 0; k < D / 16; ++k) asm volatile("" : "+v"(r[k]));
#pragma unroll
    for (int k = 0; k < D / 32; ++k) asm volatile("" : "+v"(lo[k]), "+v"(hi[k]));
  }
  __device__ __forceinline__ void flip() {
#pragma unroll
    for (int k = 0; k < D / 16; ++k) { r[k] ^= STAGE; asm volatile("" : "+v"(r[k])); }
#pragma unroll
    for (int k = 0; k < D / 32; ++k) { lo[k] ^= STAGE; hi[k] ^= STAGE; asm volatile("" : "+v"(lo[k]), "+v"(hi[k])); }
  }
  // rows [rb, rb + 32) of tile A (0) or B (1), contraction over d in [16 k, 16 k + 16)
  __device__ __forceinline__ bf16x8 rows(int tile, int rb, int k) const {
    return *(const LDS_AS bf16x8*)(uintptr_t)(r[k] + (unsigned)(tile * TILE_BYTES + rb * (D * 2)));
  }
  // d in [32 k, 32 k + 32), contraction over the 16 rows from tb on
  __device__ __forceinline__ bf16x8 cols(int tile, int k, int tb) const {
    const unsigned at = (unsigned)(tile * TILE_BYTES + tb * (D * 2));
    union { struct { s16x4 a, b; } s; bf16x8 v; } u;
    u.s.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(uintptr_t)(lo[k] + at));
    u.s.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(uintptr_t)(hi[k] + at + 8u * (D * 2)));
    return u.v;
  }
};

// fragment of 32 rows of a row-major [*, ld] matrix straight from global memory (rows = MFMA rows)
template <int D>
__device__ void load_row_frags(const bf16* __restrict__ g, int64_t ld, int row0, int nrows, bf16x8 (&f)[D / 16], int d) {
  const int lane = threadIdx.x & 63;
  const int row = row0 + (lane & 31);
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    bf16x8 val = {0, 0, 0, 0, 0, 0, 0, 0};
    const int c = kk * 16 + (lane >> 5) * 8;
    if (row < nrows && c < d) val = *reinterpret_cast<const bf16x8*>(g + (int64_t)row * ld + c);
    f[kk] = val;
  }
}

// Order hint for a run of N1 products whose LDS fragment is R1 ds_read instructions each, followed by N2 products
// with R2 reads each: the fragments of the first kAhead products are requested before the first product, then each
// product is followed by the request for the product kAhead places later.  (Left alone, the compiler waits for each
// fragment right before the product that uses it, and the matrix core idles for an LDS round trip every time.)
template <int N1, int R1, int N2 = 0, int R2 = 0>
__device__ __forceinline__ void lds_ahead_schedule() {
  constexpr int N = N1 + N2, kAhead = N1 < 4 ? N1 : 4;
  __builtin_amdgcn_sched_group_barrier(0x100, kAhead * R1, 0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (i + kAhead < N1) __builtin_amdgcn_sched_group_barrier(0x100, R1, 0);
    else if (i + kAhead < N) __builtin_amdgcn_sched_group_barrier(0x100, R2, 0);
  }
}

__device__ __forceinline__ bf16x8 pack8(const f32x16& v, int e0) {
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (bf16)v[e0 + i];
  return r;
}

// accumulator rows d (4 consecutive per group) of column token -> out[token][d0 + d], scaled
template <int D>
__device__ void store_transposed(const f32x16 (&acc)[D / 32], bf16* __restrict__ out, int64_t ld, int token, int ntokens, float mul, int d) {
  if (token >= ntokens) return;
  const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bf16x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (bf16)(acc[dt][4 * j + i] * mul);
      const int d0 = dt * 32 + 8 * j + 4 * h;
      if (d0 < d) *reinterpret_cast<bf16x4*>(out + (int64_t)token * ld + d0) = v;      // (d is a multiple of 8: a group of 4 is in or out)
    }
}

// The same store for a gradient with respect to rotated queries or keys: each pair (2i, 2i+1) is first turned back by
// the angle of its position, rot[token][i] = (cos, sin), so that what is stored is the gradient before the rotation.
template <int D>
__device__ void store_transposed_unrotated(const f32x16 (&acc)[D / 32], bf16* __restrict__ out, int64_t ld, int token, int ntokens, float mul,
                                           const float* __restrict__ rot, int d) {
  asm volatile("" : "+v"(token));      // (the addresses are formed here: formed ahead, they are held through the whole pass and spill)
  if (token >= ntokens) return;
  const int h = (threadIdx.x & 63) >> 5;
  const f32x4* cs = reinterpret_cast<const f32x4*>(rot + (int64_t)token * d);      // d/2 pairs of (cos, sin) per position
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d0 = dt * 32 + 8 * j + 4 * h;
      if (d0 >= d) continue;
      const f32x4 r = cs[d0 / 4];                                                   // pairs d0/2 and d0/2 + 1
      const float e0 = acc[dt][4 * j] * mul, o0 = acc[dt][4 * j + 1] * mul, e1 = acc[dt][4 * j + 2] * mul, o1 = acc[dt][4 * j + 3] * mul;
      bf16x4 v;
      v[0] = (bf16)(e0 * r[0] + o0 * r[1]);
      v[1] = (bf16)(o0 * r[0] - e0 * r[1]);
      v[2] = (bf16)(e1 * r[2] + o1 * r[3]);
      v[3] = (bf16)(o1 * r[2] - e1 * r[3]);
      *reinterpret_cast<bf16x4*>(out + (int64_t)token * ld + d0) = v;
    }
}

// f(0), f(1), .. f(N - 1) with the index as a type: products and what runs between them, unrolled whatever their number
template <typename F, int... I> __device__ __forceinline__ void static_steps_of(F& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F> __device__ __forceinline__ void static_steps(F f) { static_steps_of(f, std::make_integer_sequence<int, N>{}); }
// place AT of PLACES over which the work on 16 elements is spread
template <int AT, int PLACES, typename F> __device__ __forceinline__ void spread(F f) {
  if constexpr (AT >= 0 && AT < PLACES) {
#pragma unroll
    for (int e = AT * 16 / PLACES; e < (AT + 1) * 16 / PLACES; ++e) f(e);
  }
}

// One wavefront's share of a key tile in the forward: 32 queries by 64 keys.  What bounds the kernels built on it and on the two below, and how their
// products and exponentials are interleaved, stands at the kernels.
// BUF: which of the two stages `at` was made for the tile is in (0 where the caller turns `at` instead).
template <int D, int BUF = 0>
__device__ __forceinline__ void fwd_tile(const FragAddr<D>& at, const bf16x8 (&qf)[D / 16], f32x16 (&o)[D / 32], float& m_run, float& l_run, float c2,
                                         bool mask, int last) {
  constexpr int NP = D / 16, DT = D / 32, N = 4 * NP, kAhead = 3;
  // S^T of the two blocks of 32 keys, then O^T += V^T P^T of each
  auto fetch = [&](int i) -> bf16x8 {
    const int seg = i / NP, j = i % NP;
    if (seg < 2) return at.rows(2 * BUF, seg * 32, j);
    return at.cols(2 * BUF + 1, j % DT, (seg - 2) * 32 + 16 * (j / DT));
  };
  bf16x8 f[kAhead], pf[2][2];
  f32x16 s[2], zero;
#pragma unroll
  for (int e = 0; e < 16; ++e) zero[e] = 0.f;
#pragma unroll
  for (int i = 0; i < kAhead; ++i) f[i] = fetch(i);
  __builtin_amdgcn_sched_barrier(0);
  float psum = 0.f;
  float neg_m = 0.f;
  auto prob = [&](int b, int e) {
    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][e], c2, neg_m));
    s[b][e] = p;
    psum += p;
  };
  static_steps<N>([&](auto step) {
    constexpr int i = decltype(step)::value, seg = i / NP, j = i % NP;
    if constexpr (seg < 2) s[seg] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], qf[j], j == 0 ? zero : s[seg], 0, 0, 0);
    else o[j % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], pf[seg - 2][j / DT], o[j % DT], 0, 0, 0);
    if constexpr (i + kAhead < N) f[i % kAhead] = fetch(i + kAhead);
    if constexpr (i == 2 * NP - 1) {
      if (mask) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[b][e] = b * 32 + 8 * (e >> 2) + (e & 3) <= last ? s[b][e] : -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[b][e]);
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * c2;          // scores enter the exponent as s*c2 (c2 > 0)
      // Running maximum, in the log2 domain.  It is only raised when some row of the wavefront would otherwise see
      // an exponent above 8 (probabilities up to 2^8 are harmless in fp32 / bf16 and cancel in the final division);
      // raising it costs a pass over the output accumulators, and after the first tiles it is rarely needed.
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
      neg_m = (m_run == -INFINITY) ? 0.f : -m_run;
#pragma unroll
      for (int e = 0; e < 16; ++e) prob(0, e);
      pf[0][0] = pack8(s[0], 0); pf[0][1] = pack8(s[0], 8);
    }
    spread<i - 2 * NP, NP>([&](int e) { prob(1, e); });
    if constexpr (i == 3 * NP - 1) { pf[1][0] = pack8(s[1], 0); pf[1][1] = pack8(s[1], 8); }
    __builtin_amdgcn_sched_barrier(0);
  });
  l_run += psum;
}

// rowsum(dO * O) of this lane's row (row0 + lane % 32), dO's row at hand
template <int D>
__device__ __forceinline__ float row_dot(const bf16* __restrict__ O, int64_t ld, int row0, int nrows, const bf16x8 (&dof)[D / 16], int d) {
  bf16x8 of[D / 16];
  load_row_frags<D>(O, ld, row0, nrows, of, d);
  float dv = 0.f;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
    for (int e = 0; e < 8; ++e) dv = __builtin_fmaf((float)of[kk][e], (float)dof[kk][e], dv);
  return dv + __shfl_xor(dv, 32, 64);
}

// One wavefront's share of a key tile in the dQ kernel: 32 queries by 64 keys, as two blocks of 32 keys.
// between(i): run after product i.
struct Nothing { template <typename I> __device__ __forceinline__ void operator()(I) const {} };
template <int D, int BUF = 0, typename Between = Nothing>
__device__ __forceinline__ void dq_tile(const FragAddr<D>& at, const bf16x8 (&qf)[D / 16], const bf16x8 (&dof)[D / 16], f32x16 (&dq)[D / 32],
                                        float c2, float lse2, float dv, bool mask, int last, Between between = Between()) {
  constexpr int NP = D / 16, N = 6 * NP, kAhead = 3, DT = D / 32;
  auto fetch = [&](int i) -> bf16x8 {
    const int seg = i / NP, j = i % NP;
    if (seg < 4) return at.rows(2 * BUF + (seg & 1), seg / 2 * 32, j);
    return at.cols(2 * BUF, j % DT, (seg - 4) * 32 + 16 * (j / DT));
  };
  bf16x8 f[kAhead], df[2][2];
  f32x16 s[2], dp[2], zero;
#pragma unroll
  for (int e = 0; e < 16; ++e) zero[e] = 0.f;
#pragma unroll
  for (int i = 0; i < kAhead; ++i) f[i] = fetch(i);
  __builtin_amdgcn_sched_barrier(0);
  auto prob = [&](f32x16& s, int e) { s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c2, -lse2)); };
  auto hide = [&](f32x16& s, int tb) {
    if (mask) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = tb * 32 + 8 * (e >> 2) + (e & 3) <= last ? s[e] : 0.f;
    }
  };
  static_steps<N>([&](auto step) {
    constexpr int i = decltype(step)::value, seg = i / NP, j = i % NP;
    if constexpr (seg == 0 || seg == 2) s[seg / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], qf[j], j == 0 ? zero : s[seg / 2], 0, 0, 0);
    else if constexpr (seg == 1 || seg == 3) dp[seg / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], dof[j], j == 0 ? zero : dp[seg / 2], 0, 0, 0);
    else dq[j % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], df[seg - 4][j / DT], dq[j % DT], 0, 0, 0);
    if constexpr (i + kAhead < N) f[i % kAhead] = fetch(i + kAhead);
    between(step);
    spread<i - NP - 1, NP>([&](int e) { prob(s[0], e); });
    spread<i - 2 * NP - 1, NP>([&](int e) { s[0][e] *= dp[0][e] - dv; });
    if constexpr (i == 3 * NP) { hide(s[0], 0); df[0][0] = pack8(s[0], 0); df[0][1] = pack8(s[0], 8); }
    spread<i - 3 * NP - 1, NP>([&](int e) { prob(s[1], e); });
    spread<i - 4 * NP - 1, NP - 1>([&](int e) { s[1][e] *= dp[1][e] - dv; });
    if constexpr (i == 5 * NP - 1) { hide(s[1], 1); df[1][0] = pack8(s[1], 0); df[1][1] = pack8(s[1], 8); }
    __builtin_amdgcn_sched_barrier(0);
  });
}

// One wavefront's share of a query tile in the dK / dV kernels that hold their keys in registers: 64 queries by 32 keys.  st: the rows' statistics,
// -lse / scale and, `dvecs` further on, -dvec, from this half-wavefront's first row on.
template <int D, bool CAUSAL, int dvecs, int BUF = 0>
__device__ __forceinline__ void dkv_tile(const FragAddr<D>& at, const bf16x8 (&kf)[D / 16], const bf16x8 (&vf)[D / 16], f32x16 (&dk)[D / 32], f32x16 (&dvv)[D / 32],
                                         const LDS_AS float* st, float c2, int t0, int t, int qb0) {
  constexpr int NP = D / 16, DT = D / 32, N = 8 * NP, kAhead = 3;
  const int h = (threadIdx.x & 63) >> 5;
  // the products: S and dP of the first block and of the second, then dV and dK of each
  auto fetch = [&](int i) -> bf16x8 {
    const int seg = i / NP, j = i % NP;
    if (seg < 4) return at.rows(2 * BUF + (seg & 1), seg / 2 * 32, j);
    return at.cols(2 * BUF + 1 - (seg & 1), j % DT, (seg - 4) / 2 * 32 + 16 * (j / DT));
  };
  f32x16 s[2], dp[2];
  auto start = [&](f32x16& acc, int at) {           // a row's statistic is where its sums start
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 v = *reinterpret_cast<const LDS_AS f32x4*>(st + at + 8 * j);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[4 * j + i] = v[i];
    }
  };
  bf16x8 f[kAhead], pf[2][2], df[2][2];
  start(s[0], 0);
#pragma unroll
  for (int i = 0; i < kAhead; ++i) f[i] = fetch(i);
  start(dp[0], dvecs);
  __builtin_amdgcn_sched_barrier(0);
  const int seen = t - qb0 - 4 * h;                 // query rows from here on see the key
  auto hide = [&](f32x16& p, int b) {
    if (CAUSAL && t0 + 31 > qb0 + b * 32) {         // (the block touches the diagonal: wave-uniform)
#pragma unroll
      for (int e = 0; e < 16; ++e) p[e] = b * 32 + 8 * (e >> 2) + (e & 3) >= seen ? p[e] : 0.f;
    }
  };
  static_steps<N>([&](auto step) {
    constexpr int i = decltype(step)::value, seg = i / NP, j = i % NP;
    if constexpr (seg == 0 || seg == 2) s[seg / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], kf[j], s[seg / 2], 0, 0, 0);
    else if constexpr (seg == 1 || seg == 3) dp[seg / 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], vf[j], dp[seg / 2], 0, 0, 0);
    else if constexpr (seg == 4 || seg == 6) dvv[j % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], pf[(seg - 4) / 2][j / DT], dvv[j % DT], 0, 0, 0);
    else dk[j % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], df[(seg - 4) / 2][j / DT], dk[j % DT], 0, 0, 0);
    if constexpr (i + kAhead < N) f[i % kAhead] = fetch(i + kAhead);
    if constexpr (i == NP) start(s[1], 32);
    if constexpr (i == 2 * NP) start(dp[1], dvecs + 32);
    // P = exp2(c2 (S - lse / scale)) and dS = P (dP - dvec)
    spread<i - NP - 1, NP>([&](int e) { s[0][e] = __builtin_amdgcn_exp2f(s[0][e] * c2); });
    if constexpr (i == 2 * NP) hide(s[0], 0);
    spread<i - 2 * NP - 1, NP - 1>([&](int e) { dp[0][e] *= s[0][e]; });
    if constexpr (i == 3 * NP - 1) {
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) { pf[0][jj] = pack8(s[0], 8 * jj); df[0][jj] = pack8(dp[0], 8 * jj); }
    }
    spread<i - 3 * NP, NP>([&](int e) { s[1][e] = __builtin_amdgcn_exp2f(s[1][e] * c2); });
    if constexpr (i == 4 * NP - 1) hide(s[1], 1);
    spread<i - 4 * NP - 1, NP - 1>([&](int e) { dp[1][e] *= s[1][e]; });
    if constexpr (i == 5 * NP - 1) {
#pragma unroll
      for (int jj = 0; jj < 2; ++jj) { pf[1][jj] = pack8(s[1], 8 * jj); df[1][jj] = pack8(dp[1], 8 * jj); }
    }
    __builtin_amdgcn_sched_barrier(0);
  });
}

}  // namespace
}  // namespace cephalo
