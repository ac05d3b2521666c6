// Rotary positions with several axes: pair (2i, 2i+1) of a head is turned by position[row][axis of the pair] * base^(-2 i' / width of the axis), i' its place
// among the axis's pairs.
//
// What bounds it is memory: every element is read and written once (6.0 TB/s on 335 MB).  A thread keeps one 16-byte chunk of a head and takes several heads of a row, whose
// angles are the same: it forms the chunk's sines and cosines once.  An angle is formed in 64 bits as a number of revolutions, reduced to its
// fraction and only then rounded: in 32 bits a position of 500 000 is a sixteenth of a radian off.
#include "positions.h"

namespace cephalo {
namespace {

template <typename T, int HEADS, bool STREAM>
__global__ void __launch_bounds__(256)
rotary_axes_kernel(RotaryAxes r, const T* src, T* dst, const int* __restrict__ positions, int64_t rows, int chunks, int parts, int rows_per_block) {      // (src may be dst)
  constexpr int V = Vec<T>::N, PAIRS = V / 2;
  const int per_row = chunks * parts, in_block = threadIdx.x / per_row, rest = threadIdx.x % per_row;
  const int64_t row = (int64_t)blockIdx.x * rows_per_block + in_block;
  if (in_block >= rows_per_block || row >= rows) return;
  const int part = rest / chunks, c = rest % chunks, pair0 = c * PAIRS;
  float cosv[PAIRS], sinv[PAIRS];
#pragma unroll
  for (int i = 0; i < PAIRS; ++i) {
    const int pair = min(pair0 + i, r.pairs - 1);
    const double turns = (double)positions[row * r.axes + r.axis[pair]] * r.turns[pair];
    sincospif(2.0f * (float)(turns - rint(turns)), &sinv[i], &cosv[i]);
  }
  for (int head0 = part; head0 < r.heads; head0 += parts * HEADS) {
    float x[HEADS][V];
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
      const int head = head0 + k * parts < r.heads ? head0 + k * parts : head0;      // (of its own heads: another's may be written meanwhile)
      load_vec<T>(src + row * r.src_pitch + head * r.d + c * V, x[k]);
    }
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
      const int head = head0 + k * parts;
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) {
        const float e = x[k][2 * i], o = x[k][2 * i + 1];
        if (pair0 + i < r.pairs) {                        // (columns past the axes' stay as they are)
          x[k][2 * i] = e * cosv[i] - o * sinv[i];
          x[k][2 * i + 1] = e * sinv[i] + o * cosv[i];
        }
      }
      if (head < r.heads) store_vec_past<T, STREAM>(dst + row * r.dst_pitch + head * r.d + c * V, x[k]);
    }
  }
}

}  // namespace

template <typename T>
int launch_rotary_axes(const RotaryAxes& r, const T* src, T* dst, const int* positions, int64_t rows, hipStream_t s) {
  const RotarySplit split = rotary_split(r.heads, r.d, Vec<T>::N);
  const int64_t blocks = (rows + split.rows - 1) / split.rows;
  // Results beyond 32 MiB, which the L2s together do not hold, go past them: 16384 rows of 40 heads of 128 (bf16, 335 MB in and out) 61.2 -> 55.8 us, the rate
  // of a copy.
  const bool stream = (int64_t)rows * r.heads * r.d * (int64_t)sizeof(T) > (int64_t)32 << 20;
  const auto kern = stream ? rotary_axes_kernel<T, kRotaryHeads, true> : rotary_axes_kernel<T, kRotaryHeads, false>;
  kern<<<(unsigned)blocks, 256, 0, s>>>(r, src, dst, positions, rows, split.chunks, split.parts, split.rows);
  CEPHALO_CHECK_LAUNCH("rotary_axes");
  return CEPHALO_OK;
}
template int launch_rotary_axes<float>(const RotaryAxes&, const float*, float*, const int*, int64_t, hipStream_t);
template int launch_rotary_axes<bf16>(const RotaryAxes&, const bf16*, bf16*, const int*, int64_t, hipStream_t);

}  // namespace cephalo
