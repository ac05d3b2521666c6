// Rotary positions with several axes.
#pragma once
#include "kernels.h"

namespace cephalo {

constexpr int kMaxRotaryPairs = 64, kMaxAxes = 8;
struct RotaryAxes {
  int64_t src_pitch, dst_pitch;      // elements
  int heads, d, axes, pairs;         // pairs: those that are turned
  double turns[kMaxRotaryPairs];     // revolutions a position, negative for the inverse
  unsigned char axis[kMaxRotaryPairs];
};
// How a launch divides the work: 16-byte chunks of a head, threads that share a row's heads, rows of a block of 256 threads.
struct RotarySplit { int chunks, parts, rows; };
constexpr int kRotaryHeads = 4;      // heads that a thread takes at a time
inline RotarySplit rotary_split(int heads, int d, int vec) {
  const int chunks = d / vec, parts = (heads + kRotaryHeads - 1) / kRotaryHeads, p = parts * chunks > 256 ? 256 / chunks : parts;
  return {chunks, p, 256 / (p * chunks)};
}
// dst[row][head] = src[row][head] turned, all heads of d columns; positions [rows, axes]; dst may be src
template <typename T> int launch_rotary_axes(const RotaryAxes& r, const T* src, T* dst, const int* positions, int64_t rows, hipStream_t s);

}  // namespace cephalo
