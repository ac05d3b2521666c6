// What the fp32 attention kernels share: operands straight from memory, products of 16 x 16 x 16, the merge of the four wavefronts.
#pragma once
#include "kernels.h"

namespace cephalo {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int kMaxHeadDim = 128;
constexpr int kWaves = 4;

// rows of a row-major [*, ld] matrix as an operand over the head's dimensions: row r0 + l % 16, dimensions 16 p + 4 g .. + 3 of piece p
// (rows past `rows` and dimensions past d are zero).  VEC: 16-byte loads (d and ld multiples of 4, aligned base).
template <int P, bool VEC>
__device__ __forceinline__ void load_rows(const float* __restrict__ m, int64_t ld, int r0, int rows, int d, f32x4 (&f)[P]) {
  const int lane = threadIdx.x & 63, r = r0 + (lane & 15), g = lane >> 4;
  const float* p = m + (int64_t)min(r, rows - 1) * ld;
  const bool ok = r < rows;
#pragma unroll
  for (int q = 0; q < P; ++q) {
    const int c = 16 * q + 4 * g;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (VEC) {
      v = *reinterpret_cast<const f32x4*>(p + (c < d ? c : 0));
      f[q] = ok && c < d ? v : f32x4{0.f, 0.f, 0.f, 0.f};
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) if (ok && c + i < d) v[i] = p[c + i];
      f[q] = v;
    }
  }
}
// the same matrix as the first operand over 16 of its rows: element [t] of piece p is row r0 + 4 g + t, column 16 p + l % 16
template <int P>
__device__ __forceinline__ void load_cols(const float* __restrict__ m, int64_t ld, int r0, int rows, int d, f32x4 (&f)[P]) {
  const int lane = threadIdx.x & 63, g = lane >> 4, c0 = lane & 15;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int r = r0 + 4 * g + t;
    const float* p = m + (int64_t)min(r, rows - 1) * ld;
#pragma unroll
    for (int q = 0; q < P; ++q) {
      const int c = 16 * q + c0;
      const float v = p[c < d ? c : 0];
      f[q][t] = r < rows && c < d ? v : 0.f;
    }
  }
}
// D[i][j] = sum over the dimensions of a[i] b[j], both from load_rows
template <int P>
__device__ __forceinline__ f32x4 dot_rows(const f32x4 (&a)[P], const f32x4 (&b)[P]) {
  f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};      // (two chains: no product waits for the one before)
#pragma unroll
  for (int q = 0; q < P; ++q)
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[q][t], b[q][t], s[t & 1], 0, 0, 0);
  return s[0] + s[1];
}
// o[piece][i] (dimension 16 piece + 4 g + i of column j) += sum over the 16 rows of cols[..] w[row of the lane's scores]
template <int P>
__device__ __forceinline__ void add_weighted(f32x4 (&o)[P], const f32x4 (&cols)[P], f32x4 w) {
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int q = 0; q < P; ++q) o[q] = __builtin_amdgcn_mfma_f32_16x16x4f32(cols[q][t], w[t], o[q], 0, 0, 0);
}
// The same for a block on the diagonal, where some of the 16 rows are masked for some columns: a weight of zero does not silence a row
// that holds an infinity or a NaN, so such a block (rare; one branch for the wavefront) is added value by value and masked rows are left
// out.  m: the matrix the rows come from; masked(r): row r0 + r does not count for this lane's column.
template <int P, typename Masked>
__device__ __forceinline__ void add_weighted_diagonal(f32x4 (&o)[P], const f32x4 (&cols)[P], f32x4 w, const float* __restrict__ m, int64_t ld, int r0, int rows, int d,
                                                      Masked masked) {
  bool bad = false;
#pragma unroll
  for (int q = 0; q < P; ++q)
#pragma unroll
    for (int t = 0; t < 4; ++t) bad = bad || !(fabsf(cols[q][t]) < INFINITY);
  if (!__any(bad)) {
    add_weighted<P>(o, cols, w);
    return;
  }
  const int lane = threadIdx.x & 63, g = lane >> 4;
  for (int r = 0; r < 16 && r0 + r < rows; ++r) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) v = (r & 3) == i ? w[i] : v;
    v = __shfl(v, (r >> 2) * 16 + (lane & 15), 64);
    if (masked(r)) continue;
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = 16 * q + 4 * g + i;
        if (c < d) o[q][i] += v * m[(int64_t)(r0 + r) * ld + c];
      }
  }
}
// sum over the four lane groups of a column
__device__ __forceinline__ float groups_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}
__device__ __forceinline__ float groups_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
template <int P>
__device__ __forceinline__ void store_columns(float* __restrict__ out, int64_t ld, int row, int rows, int d, const f32x4 (&o)[P], float mul) {
  if (row >= rows) return;
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int q = 0; q < P; ++q)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = 16 * q + 4 * g + i;
      if (c < d) out[(int64_t)row * ld + c] = o[q][i] * mul;
    }
}
// Adds the wavefronts' `o` in wavefront order into wavefront 0's (red: W - 1 images of P x 64 lanes x 4).
template <int P, int W = kWaves>
__device__ __forceinline__ void merge_sums(f32x4 (&o)[P], f32x4* red) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  __syncthreads();
  if (wave > 0) {
#pragma unroll
    for (int q = 0; q < P; ++q) red[((wave - 1) * P + q) * 64 + lane] = o[q];
  }
  __syncthreads();
  if (wave == 0) {
#pragma unroll
    for (int w = 0; w < W - 1; ++w)
#pragma unroll
      for (int q = 0; q < P; ++q) o[q] += red[(w * P + q) * 64 + lane];
  }
}

// o[r] . do[r] of row r = r0 + l % 16, in every lane of the column; dof: those rows of dO
template <int P, bool VEC>
__device__ __forceinline__ float row_dot(const float* __restrict__ O, int64_t ld, int r0, int rows, int d, const f32x4 (&dof)[P]) {
  f32x4 of[P];
  load_rows<P, VEC>(O, ld, r0, rows, d, of);
  float v = 0.f;
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) v = fmaf(of[i][e], dof[i][e], v);
  return groups_sum(v);
}

}  // namespace
}  // namespace cephalo
